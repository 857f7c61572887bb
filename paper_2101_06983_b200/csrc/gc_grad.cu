// The global 2-norm of a list of gradients, and their clipping: what stands between Step 3 (Section 3.3,
// the full-batch gradient dL/dW summed over the sub-batches) and an optimiser.
//
//     n^2 = sum_t sum_e g_te^2        c = min(1, max_norm / (n + 1e-6))        out_te = c g_te
//
// The tensors of a list travel as kernel parameters (pointers, extents, first tile), so a call copies nothing
// to the device and can be captured.  The list is cut into tiles of 32 KB (2048 vectors; 4 or 8 KB where single
// elements take their place), dealt to the blocks in turn.
// Squares of up to 32 values are summed in fp32; a sum outside [2^-100, inf) whose values are not all zero
// (squares that overflowed, or that lost bits below 2^-149) is formed again in fp64, and everything beyond
// those 32 values is summed in fp64, in an order that the sizes alone fix.
#include <cuda_bf16.h>
#include <math.h>

#include <algorithm>
#include <vector>

#include "gc_internal.h"

namespace gc {
namespace {

constexpr int GR_THREADS = 512;
constexpr int GR_PER = 4;                      // of a thread, all under way at once
// Blocks to an SM of the two passes.  Measured, us per clipping of 357 MB fp32 / 178 MB bf16 / 666 MB bf16 with 3 and 3 blocks
// 180 / 89 / 334, 3 and 2 177 / 88 / 332, 4 and 3 180 / 89 / 336; tiles of 16 KB 188 / 95 / 370, of 64 KB 179 / 90 / 332.
constexpr int GR_B1 = 3, GR_B2 = 2;
constexpr int GR_TILE_UNITS = GR_THREADS * GR_PER;   // 16-byte vectors of a tile; single elements where they do not fit
// Lists of at most so many tiles take one launch of a cluster instead of two of the whole device.  Measured, us a call back to
// back from the host, then in a graph, 8 tiles: norm 5.0 and 3.4 (two launches 7.0 and 3.2), clipping 5.3 and 5.4 (7.0
// and 4.6); 16 tiles: clipping 5.5 and 5.5 (7.1 and 4.8); 36, in a cluster of 16: 7.8 and 7.7 (7.1 and 4.9).
constexpr uint32_t GR_SHORT = 16;
constexpr int GR_CLUSTER = 8;                  // two tiles to a CTA
static_assert(2 * GR_CLUSTER >= GR_SHORT, "the largest cluster takes the longest short list in a round");
constexpr int GR_SLOTS = 1024;                 // partial sums of a launch
constexpr double GR_EPS = 1e-6;
// Elements of a list: its tiles, of 2^11 single elements at least but for one of each tensor, and the strides that kernels
// add to their indices stay below 2^32.
constexpr int64_t GR_MOST = (int64_t)1 << 42;

// FLAT_VEC: one stretch, vectors but for a few elements at its ends.  ROWS_VEC: rows of whole vectors.  ELEM: whatever is
// neither, among it a source and a destination on different places within 16 bytes (both passes of a clipping).
// Measured, us per 400 MB: norm of rows as vectors 93, of single elements fp32 317 and bf16 603; clipping
// into outputs alike within 16 bytes 195, one element off fp32 861 and bf16 1622.
enum EntryMode : uint32_t { FLAT_VEC = 0, ROWS_VEC = 1, ELEM = 2 };

struct Entry {
    const void* src;
    void* dst;
    int64_t units;        // FLAT_VEC, ROWS_VEC: whole vectors; ELEM: elements
    int64_t ld, ld_out;   // elements
    uint32_t cols;        // ROWS_VEC: vectors of a row; ELEM: elements of a row
    uint16_t mode;
    uint16_t bf16;
    uint16_t head, tail;  // FLAT_VEC: single elements before and after the vectors
};
template <int N>
struct List {
    int n;
    uint32_t tiles;
    uint32_t first[N];    // first tile of each entry: side by side, for the search
    Entry e[N];
};
constexpr int FEW = 32, SOME = 96, MORE = 224, MANY = 540;        // 32,764 bytes of parameters at most; fewer are copied faster
static_assert(sizeof(List<MANY>) <= 32600, "kernel parameters");

__device__ __forceinline__ float2 widen(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ uint32_t scale_pair(uint32_t w, float c) {
    const float2 v = widen(w);
    const __nv_bfloat162 r = __floats2bfloat162_rn(v.x * c, v.y * c);
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint4 scale_vec(const uint4& v, bool bf16, float c) {
    if (bf16) return make_uint4(scale_pair(v.x, c), scale_pair(v.y, c), scale_pair(v.z, c), scale_pair(v.w, c));
    return make_uint4(__float_as_uint(__uint_as_float(v.x) * c), __float_as_uint(__uint_as_float(v.y) * c),
                      __float_as_uint(__uint_as_float(v.z) * c), __float_as_uint(__uint_as_float(v.w) * c));
}
// Sum of squares of N vectors (their raw words), see the head of the file.
template <int N>
__device__ __forceinline__ double square_sum(const uint4 (&v)[N], bool bf16) {
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            any |= w[k];
            if (bf16) {
                const float2 x = widen(w[k]);
                s[k] = fmaf(x.x, x.x, s[k]);
                s[k] = fmaf(x.y, x.y, s[k]);
            } else {
                const float x = __uint_as_float(w[k]);
                s[k] = fmaf(x, x, s[k]);
            }
        }
    }
    const float t = (s[0] + s[1]) + (s[2] + s[3]);
    if (t >= 0x1p-100f && t < INFINITY) return (double)t;
    if (any == 0) return 0.0;
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 x = bf16 ? widen(w[k]) : make_float2(__uint_as_float(w[k]), 0.f);
            d = fma((double)x.x, (double)x.x, d);
            d = fma((double)x.y, (double)x.y, d);
        }
    }
    return d;
}
__device__ __forceinline__ float load_one(const void* p, int64_t i, bool bf16) {
    return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void scale_one(const Entry& e, int64_t from, int64_t to, bool copy, float c) {
    if (e.bf16) {
        const uint16_t x = static_cast<const uint16_t*>(e.src)[from];
        const __nv_bfloat16 y = __float2bfloat16_rn(__uint_as_float((uint32_t)x << 16) * c);
        static_cast<uint16_t*>(e.dst)[to] = copy ? x : *reinterpret_cast<const uint16_t*>(&y);
    } else {
        const uint32_t x = static_cast<const uint32_t*>(e.src)[from];
        static_cast<uint32_t*>(e.dst)[to] = copy ? x : __float_as_uint(__uint_as_float(x) * c);
    }
}

// The entry that holds tile t, between two that surround it.
template <int N>
__device__ __forceinline__ int entry_of(const List<N>& list, uint32_t t, int lo, int hi) {
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (list.first[mid] <= t) lo = mid; else hi = mid - 1;
    }
    return lo;
}
// Tile t of an entry that is no stretch of vectors: its first unit and where that lies.
struct Tile {
    int64_t r;
    uint32_t c, n;        // row and column of the first unit; units of the tile
};
__device__ __forceinline__ Tile tile_of(const Entry& e, uint32_t t) {
    const int64_t u = (int64_t)t * GR_TILE_UNITS;
    Tile x;
    x.n = (uint32_t)min((int64_t)GR_TILE_UNITS, e.units - u);
    x.r = u / e.cols;
    x.c = (uint32_t)(u - x.r * e.cols);
    return x;
}
// Where unit k of it lies, in elements from a base of pitch ld.
__device__ __forceinline__ int64_t place_of(const Entry& e, const Tile& x, uint32_t k, int64_t ld) {
    const uint32_t at = x.c + k, down = at / e.cols;      // (both below 2^31 + 2^10)
    return (x.r + down) * ld + (int64_t)(at - down * e.cols) * (e.mode == ROWS_VEC ? (e.bf16 ? 8 : 4) : 1);
}

__device__ __forceinline__ double warp_sum(double v) {
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Sum over the block, in every thread.
__device__ __forceinline__ double block_sum(double v, double* part) {
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) s += part[w];
    return s;
}

// A thread's share of the sum of squares of tile t of entry e (tid: of GR_THREADS).
__device__ __forceinline__ double squares_of(const Entry& e, uint32_t t, int tid) {
    const bool bf16 = e.bf16;
    uint4 v[GR_PER];
    if (e.mode == FLAT_VEC) {
        const int64_t u = (int64_t)t * GR_TILE_UNITS + tid;
        const char* src = static_cast<const char*>(e.src) + e.head * (bf16 ? 2 : 4) + 16 * u;
        if (u - tid + GR_TILE_UNITS <= e.units) {
#pragma unroll
            for (int i = 0; i < GR_PER; ++i) v[i] = *reinterpret_cast<const uint4*>(src + 16 * GR_THREADS * i);
        } else {
#pragma unroll
            for (int i = 0; i < GR_PER; ++i)
                v[i] = u + i * GR_THREADS < e.units ? *reinterpret_cast<const uint4*>(src + 16 * GR_THREADS * i)
                                                    : make_uint4(0, 0, 0, 0);
        }
        double sum = square_sum(v, bf16);
        if (t == 0 && tid < e.head + e.tail) {
            const double x = load_one(e.src, tid < e.head ? tid : tid + e.units * (bf16 ? 8 : 4), bf16);
            sum = fma(x, x, sum);
        }
        return sum;
    }
    const Tile x = tile_of(e, t);
    if (e.mode == ROWS_VEC) {
#pragma unroll
        for (int i = 0; i < GR_PER; ++i) {
            const uint32_t k = tid + i * GR_THREADS;
            v[i] = k < x.n ? *reinterpret_cast<const uint4*>(static_cast<const char*>(e.src) +
                                                             place_of(e, x, k, e.ld) * (bf16 ? 2 : 4))
                           : make_uint4(0, 0, 0, 0);
        }
        return square_sum(v, bf16);
    }
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < GR_PER; ++i) {
        const uint32_t k = tid + i * GR_THREADS;
        if (k < x.n) {
            const double y = load_one(e.src, place_of(e, x, k, e.ld), bf16);
            sum = fma(y, y, sum);
        }
    }
    return sum;
}
// out = c g (copy: out = g) for a thread's share of tile t of entry e.
__device__ __forceinline__ void scale_tile(const Entry& e, uint32_t t, int tid, bool copy, float c) {
    const bool bf16 = e.bf16;
    if (copy && e.src == e.dst) return;                  // the values stay as they are
    if (e.mode == FLAT_VEC) {
        const int64_t u = (int64_t)t * GR_TILE_UNITS + tid;
        const char* src = static_cast<const char*>(e.src) + e.head * (bf16 ? 2 : 4) + 16 * u;
        char* dst = static_cast<char*>(e.dst) + e.head * (bf16 ? 2 : 4) + 16 * u;
        if (u - tid + GR_TILE_UNITS <= e.units) {
            uint4 v[GR_PER];
#pragma unroll
            for (int i = 0; i < GR_PER; ++i) v[i] = *reinterpret_cast<const uint4*>(src + 16 * GR_THREADS * i);
#pragma unroll
            for (int i = 0; i < GR_PER; ++i)
                *reinterpret_cast<uint4*>(dst + 16 * GR_THREADS * i) = copy ? v[i] : scale_vec(v[i], bf16, c);
        } else {
#pragma unroll
            for (int i = 0; i < GR_PER; ++i)
                if (u + i * GR_THREADS < e.units) {
                    const uint4 v = *reinterpret_cast<const uint4*>(src + 16 * GR_THREADS * i);
                    *reinterpret_cast<uint4*>(dst + 16 * GR_THREADS * i) = copy ? v : scale_vec(v, bf16, c);
                }
        }
        if (t == 0 && tid < e.head + e.tail) {
            const int64_t i = tid < e.head ? tid : tid + e.units * (bf16 ? 8 : 4);
            scale_one(e, i, i, copy, c);
        }
        return;
    }
    const Tile x = tile_of(e, t);
#pragma unroll
    for (int i = 0; i < GR_PER; ++i) {
        const uint32_t k = tid + i * GR_THREADS;
        if (k >= x.n) break;
        const int64_t from = place_of(e, x, k, e.ld), to = place_of(e, x, k, e.ld_out);
        if (e.mode == ROWS_VEC) {
            const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const char*>(e.src) + from * (bf16 ? 2 : 4));
            *reinterpret_cast<uint4*>(static_cast<char*>(e.dst) + to * (bf16 ? 2 : 4)) =
                copy ? v : scale_vec(v, bf16, c);
        } else {
            scale_one(e, from, to, copy, c);
        }
    }
}

// part[block] = the sum of squares of the block's tiles.
template <int N>
__global__ void __launch_bounds__(GR_THREADS, GR_B1)
grad_square_kernel(const __grid_constant__ List<N> list, double* part) {
    __shared__ double warp_part[GR_THREADS / 32];
    dep_release();
    dep_wait();
    double sum = 0.0;
    int at = 0;
    for (uint32_t t = blockIdx.x; t < list.tiles; t += gridDim.x) {
        at = entry_of(list, t, at, list.n - 1);
        sum += squares_of(list.e[at], t - list.first[at], threadIdx.x);
    }
    sum = block_sum(sum, warp_part);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// The sum of `slots` partial sums, in every thread of the block.
__device__ __forceinline__ double total_of(const double* part, int slots, double* warp_part) {
    double s = 0.0;
    for (int i = threadIdx.x; i < slots; i += blockDim.x) s += __ldcg(part + i);
    return block_sum(s, warp_part);
}
__device__ __forceinline__ void tell_norm(double total, double* sq_sum, float* norm, int* dev_status) {
    if (sq_sum) *sq_sum = total;
    if (norm) *norm = (float)sqrt(total);
    if (dev_status && !isfinite(sqrt(total))) atomicOr(dev_status, GC_DEV_GRAD_NONFINITE);
}

// The factor of the gradients.  *copy: it is 1 or more, or the sum not finite, and values are copied bit for bit, a NaN's
// payload too (told from the fp64 factor: by c == 1 the compiler takes a product with c for the same).
__device__ __forceinline__ float factor_of(double total, float max_norm, bool* copy) {
    const double norm = sqrt(total), wide = (double)max_norm / (norm + GR_EPS);
    *copy = !isfinite(norm) || wide >= 1.0;
    return (float)wide;
}

__global__ void __launch_bounds__(GR_THREADS)
grad_norm_kernel(const double* part, int slots, double* sq_sum, float* norm, int* dev_status) {
    __shared__ double warp_part[GR_THREADS / 32];
    dep_release();
    dep_wait();
    const double total = total_of(part, slots, warp_part);
    if (threadIdx.x == 0) tell_norm(total, sq_sum, norm, dev_status);
}

// out = c g, c from the sum of `slots` partial sums.
template <int N>
__global__ void __launch_bounds__(GR_THREADS, GR_B2)
grad_scale_kernel(const __grid_constant__ List<N> list, const double* part, int slots, float max_norm,
                  double* sq_sum, float* norm, int* dev_status, int tell) {
    __shared__ double warp_part[GR_THREADS / 32];
    dep_release();
    dep_wait();
    const double total = total_of(part, slots, warp_part);
    if (tell && blockIdx.x == 0 && threadIdx.x == 0) tell_norm(total, sq_sum, norm, dev_status);
    bool copy;
    const float c = factor_of(total, max_norm, &copy);
    // backwards: what the sum of squares read last is in the L2 still
    int at = list.n - 1;
    for (int64_t back = (int64_t)list.tiles - 1 - blockIdx.x; back >= 0; back -= gridDim.x) {
        const uint32_t t = (uint32_t)back;
        at = entry_of(list, t, 0, at);
        scale_tile(list.e[at], t - list.first[at], threadIdx.x, copy, c);
    }
}

// Short lists: both passes in one cluster, whose CTAs exchange their sums through shared memory.  Two halves of a CTA
// take a tile each.
template <int N, bool CLIP>
__global__ void __launch_bounds__(2 * GR_THREADS, 1)
grad_cluster_kernel(const __grid_constant__ List<N> list, float max_norm, double* sq_sum, float* norm, int* dev_status) {
    __shared__ double warp_part[2 * GR_THREADS / 32];
    __shared__ double sums[GR_CLUSTER];
    const int tid = threadIdx.x % GR_THREADS, ctas = gridDim.x;
    const uint32_t first = 2 * blockIdx.x + threadIdx.x / GR_THREADS, by = 2 * ctas;
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // this CTA has started
    dep_release();
    dep_wait();
    double sum = 0.0;
    int at = 0;
    for (uint32_t t = first; t < list.tiles; t += by) {
        at = entry_of(list, t, at, list.n - 1);
        sum += squares_of(list.e[at], t - list.first[at], tid);
    }
    sum = block_sum(sum, warp_part);
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");                // and so have those it sends to
    if ((int)threadIdx.x < ctas) {
        uint32_t there;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                     : "=r"(there) : "r"((uint32_t)__cvta_generic_to_shared(&sums[blockIdx.x])), "r"(threadIdx.x));
        asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(there), "d"(sum) : "memory");
    }
    asm volatile("barrier.cluster.arrive.release.aligned;\n\t"
                 "barrier.cluster.wait.acquire.aligned;" ::: "memory");
    double total = 0.0;
    for (int i = 0; i < ctas; ++i) total += sums[i];
    if (blockIdx.x == 0 && threadIdx.x == 0) tell_norm(total, sq_sum, norm, dev_status);
    if (!CLIP) return;
    bool copy;
    const float c = factor_of(total, max_norm, &copy);
    for (uint32_t t = first; t < list.tiles; t += by) {
        at = entry_of(list, t, 0, list.n - 1);
        scale_tile(list.e[at], t - list.first[at], tid, copy, c);
    }
}

// ---- host ------------------------------------------------------------------------------------------
// The bytes from a tensor's first to its last, at one of its two places.
struct Span {
    uintptr_t lo, hi;
    int64_t pitch;        // bytes from row to row; 0: one row
    int64_t width;        // bytes of a row
    bool written;
};

int elem_size(int dtype) { return dtype == GC_BF16 ? 2 : 4; }

// Checks one tensor; *count its elements.
int check_tensor(const gc_tensor& t, bool write, int64_t* count) {
    if (t.dtype != GC_F32 && t.dtype != GC_BF16) return GC_ERR_DTYPE;
    if (t.rows < 0 || t.cols < 0) return GC_ERR_SHAPE;
    *count = 0;
    if (t.rows == 0 || t.cols == 0) return GC_OK;
    const int64_t limit = (int64_t)1 << 40;
    if (t.cols > limit || t.rows > limit / t.cols) return GC_ERR_SHAPE;
    if (t.rows > 1 && t.cols > ((int64_t)1 << 31)) return GC_ERR_LIMIT;
    if (t.rows > 1 && (t.ld < t.cols || t.ld > limit || t.rows > ((int64_t)1 << 60) / t.ld)) return GC_ERR_SHAPE;
    if (!t.data) return GC_ERR_NULL;
    const uintptr_t es = (uintptr_t)elem_size(t.dtype);
    if ((uintptr_t)t.data % es) return GC_ERR_ALIGN;
    if (write && t.out && t.out != t.data) {
        if (t.rows > 1 && (t.ld_out < t.cols || t.ld_out > limit || t.rows > ((int64_t)1 << 60) / t.ld_out))
            return GC_ERR_SHAPE;
        if ((uintptr_t)t.out % es) return GC_ERR_ALIGN;
    }
    *count = t.rows * t.cols;
    return GC_OK;
}
uintptr_t bytes_of(const gc_tensor& t, int64_t ld) {
    return (uintptr_t)(((t.rows - 1) * ld + t.cols) * elem_size(t.dtype));
}
// Spans that come in ascending order, in a few strands that lie apart (tensors of flat buffers, one for each type, and
// their outputs): no two of them meet.  The usual list, told without sorting it.
struct Strands {
    static constexpr int MOST = 8;
    static constexpr uintptr_t NEAR = 1 << 16;
    uintptr_t lo[MOST], hi[MOST];
    int n = 0;
    bool good = true;
    void add(uintptr_t a, uintptr_t b) {
        for (int k = 0; k < n; ++k)
            if (a >= hi[k] && a - hi[k] < NEAR) {
                hi[k] = b;
                return;
            }
        if (n == MOST) { good = false; return; }
        lo[n] = a;
        hi[n++] = b;
    }
    bool apart() const {
        for (int i = 0; i < n && good; ++i)
            for (int k = 0; k < i; ++k)
                if (lo[i] < hi[k] && lo[k] < hi[i]) return false;
        return good;
    }
};
// How many of a set of intervals meet a given one: those that start before its end, less those that end before its start.
// Counts lie in binary indexed trees over the ends that occur.
class Intervals {
public:
    Intervals(const std::vector<int64_t>& starts, const std::vector<int64_t>& ends)
        : starts_(starts), ends_(ends), n_starts_(starts.size() + 1), n_ends_(ends.size() + 1) {}
    void add(int64_t a, int64_t b, int by) {
        for (size_t i = below(starts_, a) + 1; i < n_starts_.size(); i += i & (~i + 1)) n_starts_[i] += by;
        for (size_t i = below(ends_, b) + 1; i < n_ends_.size(); i += i & (~i + 1)) n_ends_[i] += by;
    }
    bool meet(int64_t a, int64_t b) const {
        int64_t n = 0;
        for (size_t i = below(starts_, b); i > 0; i &= i - 1) n += n_starts_[i];
        for (size_t i = below(ends_, a + 1); i > 0; i &= i - 1) n -= n_ends_[i];
        return n > 0;
    }

private:
    static size_t below(const std::vector<int64_t>& v, int64_t x) { return std::lower_bound(v.begin(), v.end(), x) - v.begin(); }
    const std::vector<int64_t>&starts_, &ends_;            // ascending, each value once
    std::vector<int64_t> n_starts_, n_ends_;
};

// Goes through n spans in ascending order of their starts: drop(i) for those that end before the next starts, then
// take(i), which is false where span i shares a place with one that has not been dropped.  False where any take is.
template <typename Drop, typename Take>
bool in_turn(const Span* s, size_t n, Drop drop, Take take) {
    std::vector<size_t> by_end(n);
    for (size_t i = 0; i < n; ++i) by_end[i] = i;
    std::sort(by_end.begin(), by_end.end(), [&](size_t a, size_t b) { return s[a].hi < s[b].hi; });
    size_t gone = 0;
    for (size_t i = 0; i < n; ++i) {
        for (; s[by_end[gone]].hi <= s[i].lo; ++gone) drop(by_end[gone]);     // (spans are not empty: i itself ends later)
        if (!take(i)) return false;
    }
    return true;
}

// Whether rows of one pitch, and single rows among them, share no place that is written.  Where two spans meet, one starts
// inside the other, and its first row shares a byte with the other's row there or the next exactly if the rows'
// intervals modulo the pitch meet.
bool rows_apart(const std::vector<Span>& s, int64_t pitch) {
    struct Piece { int64_t a, b; };
    std::vector<Piece> pieces(2 * s.size());               // the interval, and what of it passes the pitch's end
    std::vector<int64_t> starts, ends;
    for (size_t i = 0; i < s.size(); ++i) {
        const int64_t a = (int64_t)(s[i].lo % (uintptr_t)pitch), b = a + std::min(s[i].width, pitch);
        pieces[2 * i] = {a, std::min(b, pitch)};
        pieces[2 * i + 1] = {0, std::max<int64_t>(0, b - pitch)};
    }
    for (const Piece& x : pieces) {
        starts.push_back(x.a);
        ends.push_back(x.b);
    }
    for (auto* v : {&starts, &ends}) {
        std::sort(v->begin(), v->end());
        v->erase(std::unique(v->begin(), v->end()), v->end());
    }
    Intervals all(starts, ends), written(starts, ends);
    auto count = [&](size_t i, int by) {
        for (size_t k = 2 * i; k < 2 * i + 2; ++k)
            if (pieces[k].a < pieces[k].b) {
                all.add(pieces[k].a, pieces[k].b, by);
                if (s[i].written) written.add(pieces[k].a, pieces[k].b, by);
            }
    };
    return in_turn(s.data(), s.size(), [&](size_t i) { count(i, -1); }, [&](size_t i) {
        const Intervals& others = s[i].written ? all : written;
        for (size_t k = 2 * i; k < 2 * i + 2; ++k)
            if (pieces[k].a < pieces[k].b && others.meet(pieces[k].a, pieces[k].b)) return false;
        count(i, 1);
        return true;
    });
}
// Whether n spans (ascending starts) share no place that is written.  Matrices of two pitches that meet count as if they did.
bool spans_apart(const Span* s, size_t n) {
    std::vector<int64_t> pitches;                          // 0, for single rows, among them
    for (size_t i = 0; i < n; ++i) pitches.push_back(s[i].pitch);
    std::sort(pitches.begin(), pitches.end());
    pitches.erase(std::unique(pitches.begin(), pitches.end()), pitches.end());
    struct Count { int64_t all = 0, written = 0; } rows;   // of matrices, whatever their pitch
    std::vector<Count> of(pitches.size());
    auto at = [&](size_t i) -> Count& {
        return of[std::lower_bound(pitches.begin(), pitches.end(), s[i].pitch) - pitches.begin()];
    };
    auto count = [&](size_t i, int by) {
        for (Count* c : {&at(i), s[i].pitch ? &rows : nullptr})
            if (c) {
                c->all += by;
                c->written += s[i].written ? by : 0;
            }
    };
    if (!in_turn(s, n, [&](size_t i) { count(i, -1); }, [&](size_t i) {
            const Count& same = at(i);
            const int64_t all = s[i].pitch ? rows.all - same.all : same.all;
            const int64_t written = s[i].pitch ? rows.written - same.written : same.written;
            count(i, 1);
            return (s[i].written ? all : written) == 0;
        }))
        return false;
    for (const int64_t pitch : pitches)
        if (pitch) {
            std::vector<Span> some;
            for (size_t i = 0; i < n; ++i)
                if (s[i].pitch == 0 || s[i].pitch == pitch) some.push_back(s[i]);
            if (!rows_apart(some, pitch)) return false;
        }
    return true;
}
// No place that is written may be read or written through another tensor of the list.
int check_overlap(const gc_tensor* list, int64_t n) {
    Strands strands;
    bool elsewhere = false;
    for (int64_t i = 0; i < n; ++i)
        if (list[i].rows > 0 && list[i].cols > 0) {
            const gc_tensor& t = list[i];
            const bool in_place = !t.out || t.out == t.data;
            if (in_place && t.out && t.rows > 1 && t.ld_out != t.ld) return GC_ERR_ALIAS;
            if (strands.good) {
                const uintptr_t lo = (uintptr_t)t.data;
                strands.add(lo, lo + bytes_of(t, t.ld));
                if (!in_place) strands.add((uintptr_t)t.out, (uintptr_t)t.out + bytes_of(t, t.ld_out));
            }
            elsewhere |= !in_place;
        }
    if (strands.apart()) return GC_OK;
    std::vector<Span> s;
    s.reserve((size_t)n * (elsewhere ? 2 : 1));
    for (int64_t i = 0; i < n; ++i)
        if (list[i].rows > 0 && list[i].cols > 0) {
            const gc_tensor& t = list[i];
            const bool in_place = !t.out || t.out == t.data;
            auto add = [&](const void* p, int64_t ld, bool written) {
                const uintptr_t lo = (uintptr_t)p;
                const int64_t es = elem_size(t.dtype);
                s.push_back({lo, lo + bytes_of(t, ld), t.rows > 1 ? ld * es : 0, t.cols * es, written});
            };
            add(t.data, t.ld, in_place);
            if (!in_place) add(t.out, t.ld_out, true);
        }
    std::sort(s.begin(), s.end(), [](const Span& a, const Span& b) { return a.lo < b.lo; });
    // stretches of spans that meet, one after the other
    for (size_t i = 0, j; i < s.size(); i = j) {
        uintptr_t end = s[i].hi;
        for (j = i + 1; j < s.size() && s[j].lo < end; ++j) end = std::max(end, s[j].hi);
        if (j - i > 1 && !spans_apart(s.data() + i, j - i)) return GC_ERR_ALIAS;
    }
    return GC_OK;
}

// The tensor as an entry; *tiles what it takes.
Entry entry_for(const gc_tensor& t, bool write, int64_t* tiles) {
    Entry e{};
    const int es = elem_size(t.dtype), vec = 16 / es;
    e.src = t.data;
    e.dst = t.out ? t.out : t.data;
    e.bf16 = t.dtype == GC_BF16;
    e.ld = t.ld;
    e.ld_out = e.dst == t.data ? t.ld : t.ld_out;
    const int64_t count = t.rows * t.cols;
    const bool flat = t.rows == 1 || (t.ld == t.cols && (!write || e.ld_out == t.cols));
    const uintptr_t s16 = (uintptr_t)e.src & 15, d16 = write ? (uintptr_t)e.dst & 15 : s16;
    if (flat && s16 == d16) {
        e.mode = FLAT_VEC;
        const int64_t head = std::min<int64_t>(count, (int64_t)((16 - s16) & 15) / es);
        e.head = (uint16_t)head;
        e.units = (count - head) / vec;
        e.tail = (uint16_t)(count - head - e.units * vec);
        e.cols = 1;
    } else if (!flat && s16 == 0 && d16 == 0 && t.cols % vec == 0 && (e.ld * es) % 16 == 0 &&
               (!write || (e.ld_out * es) % 16 == 0) && t.cols / vec < ((int64_t)1 << 31)) {
        e.mode = ROWS_VEC;
        e.units = count / vec;
        e.cols = (uint32_t)(t.cols / vec);
    } else {
        e.mode = ELEM;
        e.units = count;
        e.cols = (uint32_t)t.cols;            // of several rows: at most 2^31
        if (flat) { e.cols = 1; e.ld = e.ld_out = 1; }
    }
    *tiles = std::max<int64_t>(1, (e.units + GR_TILE_UNITS - 1) / GR_TILE_UNITS);
    return e;
}

int current_device() {
    int dev = 0, major = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) {
        cudaGetLastError();
        return GC_ERR_CUDA;
    }
    return major == 10 ? GC_OK : GC_ERR_ARCH;
}

int64_t groups_of(int64_t n) { return std::max<int64_t>(1, (n + MANY - 1) / MANY); }

// The next group, of MANY tensors that are not empty or what is left of them, from tensor *i on: no list has more groups than
// groups_of its length, for which the workspace has room.
void next_group(const gc_tensor* list, int64_t n, bool write, int64_t* i, List<MANY>& l) {
    l.n = 0;
    int64_t tiles = 0;                                 // (GR_MOST bounds them)
    for (; *i < n && l.n < MANY; ++*i) {
        if (list[*i].rows == 0 || list[*i].cols == 0) continue;
        int64_t more = 0;
        Entry e = entry_for(list[*i], write, &more);
        l.first[l.n] = (uint32_t)tiles;
        tiles += more;
        l.e[l.n++] = e;
    }
    l.tiles = (uint32_t)tiles;
}
// go(list) with the smallest list type that holds the group.
template <int N, typename Go>
cudaError_t with_size(const List<MANY>& l, Go go) {
    List<N> x;
    std::copy(l.e, l.e + l.n, x.e);
    std::copy(l.first, l.first + l.n, x.first);
    x.n = l.n;
    x.tiles = l.tiles;
    return go(x);
}
template <typename Go>
int with_list(const List<MANY>& l, Go go) {
    const cudaError_t e = l.n <= FEW ? with_size<FEW>(l, go) : l.n <= SOME ? with_size<SOME>(l, go)
                          : l.n <= MORE ? with_size<MORE>(l, go) : go(l);
    if (e == cudaSuccess) return GC_OK;
    cudaGetLastError();
    return GC_ERR_CUDA;
}

unsigned grid_for(uint32_t tiles, int per_sm) {
    const uint32_t most = (uint32_t)std::min(GR_SLOTS, per_sm * sm_count());
    return std::max(1u, std::min(tiles, most));
}

int check_list(const gc_tensor* list, int64_t n, bool write) {
    if (n < 0) return GC_ERR_SHAPE;
    if (n > 0 && !list) return GC_ERR_NULL;
    if (n > (int64_t)1 << 20) return GC_ERR_LIMIT;
    int64_t all = 0;
    for (int64_t i = 0; i < n; ++i) {
        int64_t count;
        const int rc = check_tensor(list[i], write, &count);
        if (rc) return rc;
        all += count;                                  // (at most 2^20 times 2^40)
    }
    if (all > GR_MOST) return GC_ERR_LIMIT;
    return write ? check_overlap(list, n) : GC_OK;
}
int check_ws(const void* ws, size_t ws_bytes, int64_t n) {
    return !ws || ((uintptr_t)ws & 255) || ws_bytes < gc_grad_workspace_bytes(n) ? GC_ERR_WORKSPACE : GC_OK;
}

// The partial sums of a group; *slots how many there are so far.
int launch_squares(const List<MANY>& group, double* part, int* slots, cudaStream_t st) {
    if (group.tiles == 0) return GC_OK;
    return with_list(group, [&](const auto& l) {
        const unsigned grid = grid_for(l.tiles, GR_B1);
        using L = std::decay_t<decltype(l)>;
        const cudaError_t e = launch_chained(grad_square_kernel<sizeof(L::e) / sizeof(Entry)>, dim3(grid), GR_THREADS, 0,
                                             1, st, l, part + *slots);
        *slots += (int)grid;
        return e;
    });
}
int launch_scale(const List<MANY>& group, const double* part, int slots, float max_norm, double* sq_sum, float* norm,
                 int* dev_status, bool tell, cudaStream_t st) {
    return with_list(group, [&](const auto& l) {
        using L = std::decay_t<decltype(l)>;
        return launch_chained(grad_scale_kernel<sizeof(L::e) / sizeof(Entry)>, dim3(grid_for(l.tiles, GR_B2)),
                              GR_THREADS, 0, 1, st, l, part, slots, max_norm, sq_sum, norm, dev_status, tell ? 1 : 0);
    });
}
// Lists short enough for one cluster.
bool is_short(const List<MANY>& group) { return group.tiles <= GR_SHORT && group.n <= FEW; }
template <bool CLIP>
int launch_short(const List<MANY>& group, float max_norm, double* sq_sum, float* norm, int* dev_status, cudaStream_t st) {
    int ctas = 1;
    while (ctas < GR_CLUSTER && 2u * ctas < group.tiles) ctas *= 2;
    const cudaError_t e = with_size<FEW>(group, [&](const List<FEW>& l) {
        return launch_chained(grad_cluster_kernel<FEW, CLIP>, dim3(ctas), 2 * GR_THREADS, 0, ctas, st, l, max_norm, sq_sum,
                              norm, dev_status);
    });
    if (e == cudaSuccess) return GC_OK;
    cudaGetLastError();
    return GC_ERR_CUDA;
}
int scale_all(const gc_tensor* list, int64_t n, const double* part, int slots, float max_norm, double* sq_sum,
              float* norm, int* dev_status, cudaStream_t st) {
    List<MANY> group;
    int64_t i = 0;
    bool tell = true;
    do {
        next_group(list, n, true, &i, group);
        const int rc = launch_scale(group, part, slots, max_norm, sq_sum, norm, dev_status, tell, st);
        if (rc) return rc;
        tell = false;
    } while (i < n);
    return GC_OK;
}

}  // namespace
}  // namespace gc

using namespace gc;

extern "C" {

size_t gc_grad_workspace_bytes(int64_t n) {
    if (n < 0 || n > (int64_t)1 << 20) return 0;
    return (size_t)groups_of(n) * GR_SLOTS * sizeof(double);
}

int gc_grad_norm(const gc_tensor* list, int64_t n, double* sq_sum, float* norm, void* ws, size_t ws_bytes,
                 int* dev_status, void* cuda_stream) try {
    if (!norm && !sq_sum) return GC_ERR_NULL;
    int rc = check_list(list, n, false);
    if (rc || (rc = check_ws(ws, ws_bytes, n)) || (rc = current_device())) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    double* part = static_cast<double*>(ws);
    List<MANY> group;
    int64_t i = 0;
    int slots = 0;
    next_group(list, n, false, &i, group);
    if (i >= n && is_short(group)) return launch_short<false>(group, 0.f, sq_sum, norm, dev_status, st);
    if ((rc = launch_squares(group, part, &slots, st))) return rc;
    while (i < n) {
        next_group(list, n, false, &i, group);
        if ((rc = launch_squares(group, part, &slots, st))) return rc;
    }
    if (launch_chained(grad_norm_kernel, dim3(1), GR_THREADS, 0, 1, st, part, slots, sq_sum, norm, dev_status) !=
        cudaSuccess) {
        cudaGetLastError();
        return GC_ERR_CUDA;
    }
    return GC_OK;
} catch (...) {
    return GC_ERR_HOST;
}

int gc_grad_scale(const gc_tensor* list, int64_t n, const double* sq_sum, float max_norm, int* dev_status,
                  void* cuda_stream) try {
    if (!sq_sum) return GC_ERR_NULL;
    if (!(max_norm >= 0.f)) return GC_ERR_SHAPE;
    int rc = check_list(list, n, true);
    if (rc || (rc = current_device())) return rc;
    return scale_all(list, n, sq_sum, 1, max_norm, nullptr, nullptr, dev_status,
                     static_cast<cudaStream_t>(cuda_stream));
} catch (...) {
    return GC_ERR_HOST;
}

int gc_grad_clip(const gc_tensor* list, int64_t n, float max_norm, double* sq_sum, float* norm, void* ws,
                 size_t ws_bytes, int* dev_status, void* cuda_stream) try {
    if (!norm) return GC_ERR_NULL;
    if (!(max_norm >= 0.f)) return GC_ERR_SHAPE;
    int rc = check_list(list, n, true);
    if (rc || (rc = check_ws(ws, ws_bytes, n)) || (rc = current_device())) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    double* part = static_cast<double*>(ws);
    List<MANY> group;
    int64_t i = 0;
    int slots = 0;
    next_group(list, n, true, &i, group);
    if (i >= n && is_short(group)) return launch_short<true>(group, max_norm, sq_sum, norm, dev_status, st);
    if ((rc = launch_squares(group, part, &slots, st))) return rc;
    if (i >= n)                                        // the only group: its list serves both passes
        return launch_scale(group, part, slots, max_norm, sq_sum, norm, dev_status, true, st);
    while (i < n) {
        next_group(list, n, true, &i, group);
        if ((rc = launch_squares(group, part, &slots, st))) return rc;
    }
    return scale_all(list, n, part, slots, max_norm, sq_sum, norm, dev_status, st);
} catch (...) {
    return GC_ERR_HOST;
}

}  // extern "C"
