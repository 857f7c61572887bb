// The linear encoder f(s) = W s and the scores S = Q P^T in 8-bit integers, for a model that has been trained:
//
//     scale_i = max_j |x_ij| / 127      q_ij = x_ij / scale_i to the nearest integer, ties to even
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

// 16 consecutive values of a row as floats; `left` of them exist.
template <bool BF16>
__device__ __forceinline__ void load16(const char* row, int64_t k, int left, float (&x)[16]) {
    if (left >= 16) {
        if (BF16) {
            const uint4* p = reinterpret_cast<const uint4*>(row + 2 * k);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 v = p[h];
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[8 * h + 2 * e] = __uint_as_float(w[e] << 16);
                    x[8 * h + 2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
                }
            }
        } else {
            const float4* p = reinterpret_cast<const float4*>(row + 4 * k);
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const float4 v = p[h];
                x[4 * h] = v.x; x[4 * h + 1] = v.y; x[4 * h + 2] = v.z; x[4 * h + 3] = v.w;
            }
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e)
        x[e] = e >= left ? 0.f : BF16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(row)[k + e])
                                      : reinterpret_cast<const float*>(row)[k + e];
}
// The 8-bit integer of x in the low byte.  x * inv misses x / scale by less than 2^-16 (both are at most 127.5,
// inv is off by 2^-24 of itself): nearer to a border than that, the quotient is formed in fp64, where no
// two quotients of 24-bit numbers on different sides of a border are the same.
__device__ __forceinline__ uint32_t to_i8(float x, float inv, float scale, bool wide) {
    const float m = fmaf(x, inv, MAGIC);
    if (wide || fabsf(fmaf(x, inv, -(m - MAGIC))) > 0.49998f) {
        const double q = rint((double)x / (double)scale);
        return (uint32_t)(int)fmin(fmax(q, -127.0), 127.0);
    }
    return __float_as_uint(m);
}

// WARPS warps to a row; a lane holds KEEP pieces of 16 values of it in registers and reads the rest twice.
template <bool BF16, int WARPS, int KEEP>
__global__ void __launch_bounds__(QZ_THREADS)
quantize_rows_kernel(const void* X, int64_t ldx, int64_t rows, int64_t d, int8_t* q, int64_t ldq, float* scale) {
    constexpr int PER_BLOCK = QZ_THREADS / 32 / WARPS, STEP = 32 * WARPS * 16;
    __shared__ uint32_t warp_max[2][QZ_THREADS / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t k0 = 16 * (lane + 32 * (warp % WARPS));
    dep_release();
    dep_wait();
    int turn = 0;
    for (int64_t i = blockIdx.x * (int64_t)PER_BLOCK + warp / WARPS; i < rows; i += (int64_t)gridDim.x * PER_BLOCK) {
        const char* src = static_cast<const char*>(X) + i * ldx * (BF16 ? 2 : 4);
        float x[KEEP][16];
        uint32_t most = 0;                 // bits of the largest |x|: infinities and NaN above every number
        auto see = [&](const float (&v)[16]) {
#pragma unroll
            for (int e = 0; e < 16; ++e) most = max(most, __float_as_uint(v[e]) & 0x7fffffffu);
        };
#pragma unroll
        for (int c = 0; c < KEEP; ++c) {
            const int64_t k = k0 + (int64_t)c * STEP;
            load16<BF16>(src, k, (int)max((int64_t)0, min((int64_t)16, d - k)), x[c]);
        }
#pragma unroll
        for (int c = 0; c < KEEP; ++c) see(x[c]);
        for (int64_t k = k0 + (int64_t)KEEP * STEP; k < d; k += STEP) {
            float v[16];
            load16<BF16>(src, k, (int)min((int64_t)16, d - k), v);
            see(v);
        }
        most = __reduce_max_sync(0xffffffffu, most);
        if (WARPS > 1) {                   // (all rows of a block end together: one row to a block)
            if (lane == 0) warp_max[turn][warp] = most;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WARPS; ++w) most = max(most, warp_max[turn][w]);
            turn ^= 1;
        }
        const bool bad = most >= 0x7f800000u;
        const float s = bad ? __uint_as_float(0x7fc00000u) : __uint_as_float(most) / 127.f;
        const bool none = bad || s == 0.f;
        const bool wide = s < 0x1p-100f;   // 1 / s may be infinite, s itself of few bits
        const float inv = none || wide ? 0.f : 1.f / s;
        if (lane == 0 && warp % WARPS == 0) scale[i] = s;
        int8_t* dst = q + i * ldq;
        auto put = [&](int64_t k, const float (&v)[16]) {
            if (k >= d) return;
            uint32_t w[4];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                uint32_t b[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) b[e] = none ? 0u : to_i8(v[4 * g + e], inv, s, wide);
                w[g] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
            }
            if (k + 16 <= d) {
                *reinterpret_cast<uint4*>(dst + k) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (k + e < d) dst[k + e] = (int8_t)(w[e >> 2] >> (8 * (e & 3)));
            }
        };
#pragma unroll
        for (int c = 0; c < KEEP; ++c) put(k0 + (int64_t)c * STEP, x[c]);
        for (int64_t k = k0 + (int64_t)KEEP * STEP; k < d; k += STEP) {
            float v[16];
            load16<BF16>(src, k, (int)min((int64_t)16, d - k), v);
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
    int k, kblocks;
    int bn;                                // rows of A in a tile: a multiple of 16 up to 256
    int stages;
    int tiles_a, tiles_b;
    const float* a_scale;
    const float* b_scale;
    void* out;
    int64_t ldo;
    int* dev_status;
};
struct ImBars {
    uint64_t full[IM_MAX_ST];
    uint64_t empty[IM_MAX_ST];
    uint64_t acc_full[2];
    uint64_t acc_free[2];
};

// Instruction descriptor, kind::i8: signed 8-bit A and B, both K-major, 32-bit integer sums.
__device__ __forceinline__ uint32_t instr_desc_i8(int n, int m) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void mma_i8(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, bool acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 da, {%1, %4};\n\t"
        "mov.b64 db, {%2, %4};\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], da, db, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(DESC_HI), "r"(acc ? 1 : 0)
        : "memory");
}

template <bool BF16>
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
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t stage_bytes = CHUNK_BYTES + (uint32_t)p.bn * 128u;
    if (threadIdx.x == 0) {
        abort_s = 0;
        for (int s = 0; s < IM_MAX_ST; ++s) {
            mbar_init(smem_u32(&bars.full[s]), 2);
            mbar_init(smem_u32(&bars.empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&bars.acc_full[b]), 1);
            mbar_init(smem_u32(&bars.acc_free[b]), NSOFT);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(&tmem_s)), "r"((uint32_t)TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_s;
    dep_release();
    dep_wait();

    const int64_t total = (int64_t)p.tiles_a * p.tiles_b;
    // the side of fewer tiles runs fastest: its rows stay in the L2 while the other side's pass once
    auto tile_at = [&](int64_t t, int* ta, int* tb) {
        if (p.tiles_a <= p.tiles_b) { *tb = (int)(t / p.tiles_a); *ta = (int)(t - (int64_t)*tb * p.tiles_a); }
        else                        { *ta = (int)(t / p.tiles_b); *tb = (int)(t - (int64_t)*ta * p.tiles_b); }
    };

    if (warp < NPROD) {
        const bool is_b = warp == 0;       // warp 0: rows of B, warp 1: rows of A
        const uint32_t bytes = is_b ? CHUNK_BYTES : (uint32_t)p.bn * 128u;
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int64_t t = blockIdx.x; t < total && ok; t += gridDim.x) {
            int ta, tb;
            tile_at(t, &ta, &tb);
            const int row = is_b ? tb * 128 : ta * p.bn;
            for (int kb = 0; kb < p.kblocks; ++kb) {
                ok = mbar_wait(smem_u32(&bars.empty[stage]), phase ^ 1u, abort_flag);
                if (!ok) break;
                const uint32_t full = smem_u32(&bars.full[stage]);
                const uint32_t dst = smem + stage * stage_bytes + (is_b ? 0u : CHUNK_BYTES);
                if (elect_one()) {
                    mbar_expect_tx(full, bytes);
                    tma_load_2d(dst, is_b ? &mapB : &mapA, kb * IM_KB, row, full);
                }
                if (++stage == p.stages) { stage = 0; phase ^= 1u; }
            }
        }
        // every stage given back: no load and no commit is under way when the block leaves
        for (int n = 0; n < p.stages && ok; ++n) {
            ok = mbar_wait(smem_u32(&bars.empty[stage]), phase ^ 1u, abort_flag);
            if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
    } else if (warp == MMA_WARP) {
        const uint32_t idesc = instr_desc_i8(p.bn, 128);
        int stage = 0, use = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int64_t t = blockIdx.x; t < total && ok; t += gridDim.x, ++use) {
            ok = mbar_wait(smem_u32(&bars.acc_free[use & 1]), ((uint32_t)(use >> 1) & 1u) ^ 1u, abort_flag);
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
                    for (int k = 0; k < 4; ++k) mma_i8(acc, b + 2 * k, a + 2 * k, idesc, kb != 0 || k != 0);
                    tc_commit(smem_u32(&bars.empty[stage]));
                    if (kb == p.kblocks - 1) tc_commit(smem_u32(&bars.acc_full[use & 1]));
                }
                if (++stage == p.stages) { stage = 0; phase ^= 1u; }
            }
        }
    } else {
        const int q = warp & 3, half = (warp - (NPROD + 1)) >> 2;
        int use = 0;
        for (int64_t t = blockIdx.x; t < total; t += gridDim.x, ++use) {
            int ta, tb;
            tile_at(t, &ta, &tb);
            const int64_t j = (int64_t)tb * 128 + 32 * q + lane;        // this lane's row of B
            const int64_t i0 = (int64_t)ta * p.bn;
            const bool live = j < p.cols;
            const float sb = live ? p.b_scale[j] : 0.f;
            if (!mbar_wait(smem_u32(&bars.acc_full[use & 1]), (uint32_t)(use >> 1) & 1u, abort_flag)) break;
            tc_fence_after();
            const uint32_t src = tmem + (use & 1) * 256 + ((uint32_t)(32 * q) << 16);
            for (int c = 16 * half; c < p.bn; c += 32) {                // 16 rows of A at a time
                if (i0 + c >= p.rows) break;
                uint32_t v[16];
                tmem_ld16(src + c, v);
                const int64_t mine = i0 + c + (lane & 15);
                const float sa = mine < p.rows ? p.a_scale[mine] : 0.f;
                tmem_ld_wait();
                float f[16];
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    f[e] = (float)(int)v[e] * __shfl_sync(0xffffffffu, sa, e) * sb;
                if (BF16) {
                    // neighbouring lanes trade a row, so that a lane stores two neighbouring outputs
#pragma unroll
                    for (int e = 0; e < 16; e += 2) {
                        const bool odd = lane & 1;
                        const float got = __shfl_xor_sync(0xffffffffu, odd ? f[e] : f[e + 1], 1);
                        const __nv_bfloat162 w = odd ? __floats2bfloat162_rn(got, f[e + 1])
                                                     : __floats2bfloat162_rn(f[e], got);
                        const int64_t i = i0 + c + e + (odd ? 1 : 0), jj = j - (odd ? 1 : 0);
                        __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(p.out) + i * p.ldo + jj;
                        if (i < p.rows) {
                            if (jj + 1 < p.cols) *reinterpret_cast<__nv_bfloat162*>(dst) = w;
                            else if (jj < p.cols) *dst = w.x;
                        }
                    }
                } else {
                    float* dst = static_cast<float*>(p.out) + (i0 + c) * p.ldo + j;
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (live && i0 + c + e < p.rows) dst[e * p.ldo] = f[e];
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
    if (warp == MMA_WARP) {
        tc_fence_after();
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
    const bool whole = d > 1024;       // a block to a row
    cudaError_t e;
    if (dtype == GC_BF16) e = whole ? go(quantize_rows_kernel<true, 8, 2>, 1) : go(quantize_rows_kernel<true, 1, 2>, 8);
    else                  e = whole ? go(quantize_rows_kernel<false, 8, 2>, 1) : go(quantize_rows_kernel<false, 1, 2>, 8);
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
    ImParams p{};
    p.rows = rows; p.cols = cols; p.k = (int)k;
    p.kblocks = (int)((k + IM_KB - 1) / IM_KB);
    p.bn = rows >= 256 ? 256 : (int)((rows + 15) / 16 * 16);
    p.tiles_a = (int)((rows + p.bn - 1) / p.bn);
    p.tiles_b = (int)((cols + 127) / 128);
    p.stages = std::min(IM_MAX_ST, (int)((IM_SMEM - 1024) / (CHUNK_BYTES + (size_t)p.bn * 128)));
    p.a_scale = a_scale; p.b_scale = b_scale; p.out = out; p.ldo = ldo; p.dev_status = dev_status;
    CUtensorMap ma, mb;
    if (!make_map_i8(&ma, A, rows, k, lda, p.bn) || !make_map_i8(&mb, B, cols, k, ldb, 128)) return GC_ERR_CUDA;
    static bool configured_on[64] = {false};       // the attribute belongs to (kernel, device)
    if (!configured_on[dev]) {
        if (cudaFuncSetAttribute(matmul_i8_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)IM_SMEM) !=
                cudaSuccess ||
            cudaFuncSetAttribute(matmul_i8_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)IM_SMEM) !=
                cudaSuccess) {
            cudaGetLastError();
            return GC_ERR_CUDA;
        }
        configured_on[dev] = true;
    }
    const int64_t total = (int64_t)p.tiles_a * p.tiles_b;
    const dim3 grid((unsigned)std::min<int64_t>(total, sm_count()));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = out_dtype == GC_BF16
        ? launch_chained(matmul_i8_kernel<true>, grid, NTHREADS, IM_SMEM, 1, st, ma, mb, p)
        : launch_chained(matmul_i8_kernel<false>, grid, NTHREADS, IM_SMEM, 1, st, ma, mb, p);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return GC_ERR_CUDA;
    }
    return GC_OK;
}

}  // extern "C"
