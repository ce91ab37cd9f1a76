// Orthogonalized updates: X <- a X + (b A + c A^2) X with A = X X^T, a few times, on the 5th-generation tensor cores.
//
// The iteration multiplies what it is given by up to a^steps where a singular value is small, so the roundings of 16-bit operands
// would show: every number is held as a pair of fp16 values, hi + lo, 22 bits of it, and a product is hi hi + hi lo + lo hi with
// fp32 accumulators.  Numbers are scaled by powers of two so that lo stays in the normal range: X by 2^14, A and the polynomial by
// 2^13.  A and A^2 are symmetric: only tiles that reach the diagonal or lie below it are computed.
// The factor a goes onto the polynomial's diagonal, B = a I + b A + c A^2, so that the new X is one product, B X.
//
// Two forms.  Matrices of at most 128 x 256 (after transposing tall ones): one block per matrix holds X, A and B in shared memory
// through all steps.  Larger ones: three tiled products per step, their operands brought in by TMA.
#include <cuda.h>
#include <math.h>

#include "nups_tcgen05.cuh"
#include "nups_types.cuh"

namespace {

constexpr float X_SCALE = 16384.0f, A_SCALE = 8192.0f;
constexpr float FROM_XX = 1.0f / (X_SCALE * X_SCALE), FROM_AA = 1.0f / (A_SCALE * A_SCALE), FROM_BX = 1.0f / (A_SCALE * X_SCALE);

struct OrthArgs {
    const void* g;
    void* out;
    uint64_t gs, gb, os, ob;   // strides of rows and of matrices
    uint32_t rows, cols, m, n; // X is m x n, m <= n
    uint32_t steps;
    int type, tall;
    float a, b, c, eps, scale;
    DevStat* st;
};

__device__ __forceinline__ float read_value(const void* p, int type, uint64_t at)
{
    if (type == NUPS_F32) return ((const float*)p)[at];
    if (type == NUPS_BF16) return __bfloat162float(((const __nv_bfloat16*)p)[at]);
    return __half2float(((const __half*)p)[at]);
}
__device__ __forceinline__ void write_value(void* p, int type, uint64_t at, float x)
{
    if (type == NUPS_F32) ((float*)p)[at] = x;
    else if (type == NUPS_BF16) ((__nv_bfloat16*)p)[at] = __float2bfloat16_rn(x);
    else ((__half*)p)[at] = __float2half_rn(x);
}
__device__ __forceinline__ void split(float x, __half& hi, __half& lo)
{
    hi = __float2half_rn(x);
    lo = __float2half_rn(x - __half2float(hi));
}
// Eight values into eight pairs, and back.
__device__ __forceinline__ void split8(const float* v, uint4& hi, uint4& lo)
{
    uint32_t* h = (uint32_t*)&hi;
    uint32_t* l = (uint32_t*)&lo;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const __half2 a = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
        const float2 f = __half22float2(a);
        const __half2 b = __floats2half2_rn(v[2 * k] - f.x, v[2 * k + 1] - f.y);
        h[k] = *(const uint32_t*)&a;
        l[k] = *(const uint32_t*)&b;
    }
}
__device__ __forceinline__ float2 join2(uint32_t hi, uint32_t lo)
{
    const float2 a = __half22float2(*(const __half2*)&hi), b = __half22float2(*(const __half2*)&lo);
    return make_float2(a.x + b.x, a.y + b.y);
}
// Sum of the squares of N floats of any size: scaled by the power of two that brings the largest near 1, added in fp32, and only
// the sum is widened (converting every value took 30 us for 4096 x 4096).  Scaling all of a matrix by a power of two changes no bit.
template <int N> __device__ __forceinline__ double sum_of_squares(const float* v)
{
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) most = fmaxf(most, fabsf(v[i]));
    const int e = max(254 - (int)(__float_as_uint(most) >> 23), 1);      // exponent field of the factor
    const float f = __int_as_float(e << 23);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) sum = fmaf(v[i] * f, v[i] * f, sum);
    return (double)sum * __hiloint2double((1023 + 2 * (127 - e)) << 20, 0);
}
// Factors that bring a matrix whose squares sum to `sum` to X: X_SCALE / (norm + eps), which may lie outside fp32's range (zeros and a
// tiny eps gave 0 times infinity), as a power of two and the rest, applied one after the other.
__device__ __forceinline__ float2 first_factors(double sum, float eps)
{
    const double f = (double)X_SCALE / (sqrt(sum) + (double)eps);         // 2^-130 (65536 x 65536 of the largest float) to 2^163
    const float power = f > 0x1p100 ? 0x1p100f : f < 0x1p-100 ? 0x1p-60f : 1.0f;
    return make_float2(power, (float)(f / (double)power));
}
__device__ __forceinline__ double warp_sum_f64(double x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

// 32 results of each of a warp's 32 rows (one row per lane) to a row-major matrix, through shared memory so that a store covers
// one row.  at: the first row's first value.
__device__ __forceinline__ void write_rows(void* out, int type, uint64_t at, uint64_t stride, uint32_t rows, uint32_t cols, const float* v, float* tile)
{
    const uint32_t lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 32; ++j) tile[lane * 33 + j] = v[j];
    __syncwarp();
    if (lane < cols)
        for (uint32_t r = 0; r < min(rows, 32u); ++r) write_value(out, type, at + r * stride + lane, tile[r * 33 + lane]);
}

// ---------------------------------------------------------------------------------------------
// one block per matrix
// ---------------------------------------------------------------------------------------------
constexpr int SMALL_M = 128, SMALL_N = 256;
constexpr uint32_t PANEL = 128 * 128;      // bytes of 64 columns of 128 rows: the unit of the operands' layout

// Byte offset of column c of row r in an operand made of panels.
__device__ __forceinline__ uint32_t panel_at(uint32_t r, uint32_t c)
{
    return (c >> 6) * PANEL + r * 128 + ((((c & 63) >> 3) ^ (r & 7)) << 4) + (c & 7) * 2;
}

__host__ __device__ constexpr uint32_t up(uint32_t x, uint32_t to) { return (x + to - 1) / to * to; }
uint32_t small_smem(uint32_t m, uint32_t n) { return (up(n, 64) / 64 + up(m, 64) / 64) * 2 * PANEL + 1024; }

// Columns of tensor memory: the widest phase's runs; a power of two.  Reads go 32 columns at a time, up to 31 further.
__device__ __forceinline__ uint32_t small_columns(uint32_t m16, uint32_t n16)
{
    const uint32_t need = max(up(n16, 64) / 64 * m16, up(m16, 64) / 64 * n16);
    uint32_t columns = 32;
    while (columns < need) columns *= 2;
    return columns;
}

// Threads: 512 where a step's results take more than two warps per quarter of the rows (64 matrices of 100 x 100: 53 us with 256,
// 41 with 512), 256 where they do not and several blocks fit a multiprocessor (600 of 64 x 64: 97 us with 256, 127 with 512).
template <int TYPE, int SMALL_BLOCK>
__global__ void __launch_bounds__(SMALL_BLOCK) orthogonalize_small_kernel(OrthArgs a)
{
    extern __shared__ char raw[];
    __shared__ uint64_t bar_mem;
    __shared__ uint32_t tmem_mem;
    __shared__ double sums[SMALL_BLOCK / 32];
    char* base = (char*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    const uint32_t nb = up(a.n, 64) / 64, mb = up(a.m, 64) / 64;
    char* const x_hi = base;
    char* const x_lo = x_hi + nb * PANEL;
    char* const a_hi = x_lo + nb * PANEL;
    char* const a_lo = a_hi + mb * PANEL;
    const uint32_t bar = smem_address(&bar_mem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        mbar_init(bar, 1);
        mbar_init_visible();
    }
    const uint32_t m16 = up(a.m, 16), n16 = up(a.n, 16), columns = small_columns(m16, n16);
    if (warp == 0) tmem_alloc<1>(smem_address(&tmem_mem), columns);
    for (uint32_t i = threadIdx.x; i < (nb + mb) * 2 * PANEL / 16; i += SMALL_BLOCK) ((uint4*)base)[i] = make_uint4(0, 0, 0, 0);
    grid_dependency_wait();
    const char* g = (const char*)a.g + (uint64_t)blockIdx.x * a.gb * (TYPE == NUPS_F32 ? 4 : 2);
    // a warp per row, four rows' loads in flight: v[k][j] is column 2 lane + 64 k + j, zero beyond the row; row(r, v)
    auto each_row = [&](auto row) {
        for (uint32_t r0 = warp; r0 < a.rows; r0 += 4 * (SMALL_BLOCK / 32)) {
            float v[4][SMALL_N / 64][2];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int k = 0; k < SMALL_N / 64; ++k)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t r = r0 + u * (SMALL_BLOCK / 32), c = 2 * lane + 64 * k + j;
                        v[u][k][j] = r < a.rows && c < a.cols ? read_value(g, TYPE, (uint64_t)r * a.gs + c) : 0.0f;
                    }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (r0 + u * (SMALL_BLOCK / 32) < a.rows) row(r0 + u * (SMALL_BLOCK / 32), v[u]);
        }
    };
    double sum = 0;
    each_row([&](uint32_t, const float (&v)[SMALL_N / 64][2]) { sum += sum_of_squares<SMALL_N / 32>(&v[0][0]); });
    sum = warp_sum_f64(sum);
    if (lane == 0) sums[warp] = sum;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_mem;
    sum = 0;
#pragma unroll
    for (int w = 0; w < SMALL_BLOCK / 32; ++w) sum += sums[w];
    const float2 f = first_factors(sum, a.eps);
    each_row([&](uint32_t r, const float (&v)[SMALL_N / 64][2]) {
#pragma unroll
        for (int k = 0; k < SMALL_N / 64; ++k) {
            const uint32_t c = 2 * lane + 64 * k;
            if (c >= a.cols) continue;                      // what is beyond the matrix is zero, as it was
            const float x = v[k][0] * f.x * f.y, y = v[k][1] * f.x * f.y;
            const __half2 hi = __floats2half2_rn(x, y);
            const float2 h = __half22float2(hi);
            const __half2 lo = __floats2half2_rn(x - h.x, y - h.y);
            if (!a.tall) {
                const uint32_t at = panel_at(r, c);
                *(__half2*)(x_hi + at) = hi;
                *(__half2*)(x_lo + at) = lo;
            } else {
                const uint32_t at = panel_at(c, r), next = panel_at(c + 1, r);
                *(__half*)(x_hi + at) = __low2half(hi);
                *(__half*)(x_lo + at) = __low2half(lo);
                if (c + 1 < a.cols) {
                    *(__half*)(x_hi + next) = __high2half(hi);
                    *(__half*)(x_lo + next) = __high2half(lo);
                }
            }
        }
    });
    const uint32_t quarter = (warp & 3) * 32, row = quarter + lane;       // tensor-memory lanes that this warp may read
    const uint32_t sxh = smem_address(x_hi), sxl = smem_address(x_lo), sah = smem_address(a_hi), sal = smem_address(a_lo);
    uint32_t phase = 0;
    bool dead = false;

    // The products of one phase.  As in the tiled kernel each run of 64 values of K (four products) has accumulators of its own,
    // `width` columns further, the small products hi lo and lo hi first; sum() adds the runs with rounding.
    auto issue = [&](uint32_t ah, uint32_t al, uint32_t bh, uint32_t bl, bool mn_major, uint32_t width, uint32_t k16) {
        if (threadIdx.x == 0) {
            tc_fence_after();
            const uint32_t shape = product_shape<1>((int)width, mn_major);
            for (int term = 0; term < 3; ++term) {
                const uint32_t pa = term == 1 ? al : ah, pb = term == 0 ? bl : bh;
                for (uint32_t k = 0; k < k16; ++k) {
                    const uint64_t da = operand_k_major(pa + (k >> 2) * PANEL + (k & 3) * 32);
                    const uint64_t db = mn_major ? operand_mn_major(pb + k * 2048, PANEL) : operand_k_major(pb + (k >> 2) * PANEL + (k & 3) * 32);
                    tc_product<1>(tmem + (k >> 2) * width, da, db, shape, term > 0 || (k & 3) > 0);
                }
            }
            tc_commit<1>(bar);
        }
        const bool ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar, phase & 1));
        ++phase;
        tc_fence_after();
        return ok;
    };
    auto sum_runs = [&](uint32_t c0, uint32_t width, uint32_t k16, float (&v)[32]) {
        __syncwarp();
        tmem_load32(tmem + (quarter << 16) + c0, v);
        for (uint32_t r = 1; r < (k16 + 3) / 4; ++r) {
            float w[32];
            tmem_load32(tmem + (quarter << 16) + r * width + c0, w);
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += w[j];
        }
    };
    // 32 columns of pairs into an operand
    auto keep = [&](char* hi_base, char* lo_base, uint32_t c0, uint32_t width, const float (&v)[32]) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (c0 + 8 * k < width) {
                uint4 hi, lo;
                split8(v + 8 * k, hi, lo);
                const uint32_t at = panel_at(row, c0 + 8 * k);
                *(uint4*)(hi_base + at) = hi;
                *(uint4*)(lo_base + at) = lo;
            }
        }
    };
    async_proxy_fence();
    __syncthreads();
    for (uint32_t step = 0; step < a.steps; ++step) {
        // A = X X^T
        bool ok = issue(sxh, sxl, sxh, sxl, false, m16, n16 / 16);
        for (uint32_t c0 = (warp >> 2) * 32; c0 < m16; c0 += SMALL_BLOCK / 4) {
            float v[32];
            sum_runs(c0, m16, n16 / 16, v);
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] *= FROM_XX * A_SCALE;
            keep(a_hi, a_lo, c0, m16, v);
        }
        tc_fence_before();
        async_proxy_fence();
        if (__syncthreads_or(!ok)) { dead = true; break; }
        // B = a I + b A + c A^2, in A's place once the products have read it
        ok = issue(sah, sal, sah, sal, false, m16, m16 / 16);
        for (uint32_t c0 = (warp >> 2) * 32; c0 < m16; c0 += SMALL_BLOCK / 4) {
            float v[32];
            sum_runs(c0, m16, m16 / 16, v);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (c0 + 8 * k < m16) {
                    const uint32_t at = panel_at(row, c0 + 8 * k);
                    const uint4 hi = *(const uint4*)(a_hi + at), lo = *(const uint4*)(a_lo + at);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 old = join2(((const uint32_t*)&hi)[j], ((const uint32_t*)&lo)[j]);
                        const uint32_t c = c0 + 8 * k + 2 * j;
                        float *x = v + 8 * k + 2 * j, diagonal = row < a.m ? a.a * A_SCALE : 0.0f;
                        x[0] = a.b * old.x + a.c * (x[0] * (FROM_AA * A_SCALE)) + (c == row ? diagonal : 0.0f);
                        x[1] = a.b * old.y + a.c * (x[1] * (FROM_AA * A_SCALE)) + (c + 1 == row ? diagonal : 0.0f);
                    }
                }
            }
            keep(a_hi, a_lo, c0, m16, v);
        }
        tc_fence_before();
        async_proxy_fence();
        if (__syncthreads_or(!ok)) { dead = true; break; }
        // X = B X
        ok = issue(sah, sal, sxh, sxl, true, n16, m16 / 16);
        const bool last = step + 1 == a.steps;
        char* out = (char*)a.out + (uint64_t)blockIdx.x * a.ob * (TYPE == NUPS_F32 ? 4 : 2);
        for (uint32_t c0 = (warp >> 2) * 32; c0 < n16; c0 += SMALL_BLOCK / 4) {
            float v[32];
            sum_runs(c0, n16, m16 / 16, v);
            if (last) {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = v[j] * FROM_BX * a.scale;       // their product may be below the normal range
                if (!ok || quarter >= a.m || c0 >= a.n) continue;          // ok: the same for all threads but after a second's wait in vain
                if (!a.tall) {
                    write_rows(out, TYPE, (uint64_t)quarter * a.os + c0, a.os, a.m - quarter, a.n - c0, v, (float*)base + warp * 32 * 33);
                } else if (row < a.m) {
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (c0 + j < a.n) write_value(out, TYPE, (uint64_t)(c0 + j) * a.os + row, v[j]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] *= FROM_BX * X_SCALE;
                keep(x_hi, x_lo, c0, n16, v);
            }
        }
        tc_fence_before();
        async_proxy_fence();
        if (__syncthreads_or(!ok)) { dead = true; break; }
    }
    if (dead && threadIdx.x == 0) atomicCAS(&a.st->status, 0, NUPS_ETIMEOUT);
    tc_fence_after();
    __syncthreads();
    if (warp == 0) tmem_free<1>(tmem, columns);
}

}  // namespace

// ---------------------------------------------------------------------------------------------
// tiled products
// ---------------------------------------------------------------------------------------------
namespace {

constexpr uint32_t NORM_RUN = 1024;        // values of a row that a block squares at a time
// Blocks that sum the squares of one matrix.
uint32_t norm_parts(uint32_t rows, uint32_t cols)
{
    const uint64_t runs = (uint64_t)rows * ((cols + NORM_RUN - 1) / NORM_RUN), parts = (runs + 7) / 8;
    return parts > 512 ? 512 : (uint32_t)parts;
}

// Where the larger matrices' pairs lie: planes of fp16 values, hi then lo, per matrix; rows padded to 16 bytes.
struct Planes {
    __half *x[2], *a, *b;
    double* sums;              // [batch][parts]
    uint32_t parts;
    float* part;               // the Gram matrix's slices
    uint32_t ldx, lda, slices;
};

__global__ void __launch_bounds__(256) orth_squares_kernel(OrthArgs a, double* sums)
{
    __shared__ double part[8];
    grid_dependency_wait();
    const char* g = (const char*)a.g + (uint64_t)blockIdx.y * a.gb * (a.type == NUPS_F32 ? 4 : 2);
    const uint32_t per_row = (a.cols + NORM_RUN - 1) / NORM_RUN;
    const uint64_t runs = (uint64_t)a.rows * per_row;
    double sum = 0;
    for (uint64_t run = blockIdx.x; run < runs; run += 4 * (uint64_t)gridDim.x) {
        float x[16];
#pragma unroll
        for (int u = 0; u < 4; ++u) {                       // four runs' loads in flight
            const uint64_t i = run + u * (uint64_t)gridDim.x;
            const uint32_t r = (uint32_t)(i / per_row), c = (uint32_t)(i % per_row) * NORM_RUN + threadIdx.x;
#pragma unroll
            for (int k = 0; k < 4; ++k) x[4 * u + k] = i < runs && c + 256 * k < a.cols ? read_value(g, a.type, (uint64_t)r * a.gs + c + 256 * k) : 0.0f;
        }
        sum += sum_of_squares<16>(x);
    }
    sum = warp_sum_f64(sum);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0;
        for (int w = 0; w < 8; ++w) sum += part[w];
        sums[blockIdx.y * gridDim.x + blockIdx.x] = sum;
    }
}

// X's first pairs, 64 x 64 values per block of 256 threads; tall matrices are transposed through shared memory.
__global__ void __launch_bounds__(256) orth_split_kernel(OrthArgs a, Planes p)
{
    __shared__ float tile[64][65];
    __shared__ double part[8];
    grid_dependency_wait();
    const char* g = (const char*)a.g + (uint64_t)blockIdx.z * a.gb * (a.type == NUPS_F32 ? 4 : 2);
    const uint32_t r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, tx = threadIdx.x & 63, ty = threadIdx.x >> 6;      // of X
    float v[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const uint32_t gr = (a.tall ? c0 : r0) + ty + 4 * k, gc = (a.tall ? r0 : c0) + tx;
        v[k] = gr < a.rows && gc < a.cols ? read_value(g, a.type, (uint64_t)gr * a.gs + gc) : 0.0f;
    }
    double sum = 0;
    for (uint32_t k = threadIdx.x; k < p.parts; k += 256) sum += p.sums[blockIdx.z * p.parts + k];
    sum = warp_sum_f64(sum);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
    if (a.tall)
#pragma unroll
        for (int k = 0; k < 16; ++k) tile[tx][ty + 4 * k] = v[k];
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) sum += part[w];
    const float2 f = first_factors(sum, a.eps);
    __half* hi = p.x[0] + (uint64_t)blockIdx.z * 2 * a.m * p.ldx;
    __half* lo = hi + (uint64_t)a.m * p.ldx;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const uint32_t r = r0 + ty + 4 * k, c = c0 + tx;
        if (r < a.m && c < a.n) {
            __half h, l;
            split((a.tall ? tile[ty + 4 * k][tx] : v[k]) * f.x * f.y, h, l);
            hi[(uint64_t)r * p.ldx + c] = h;
            lo[(uint64_t)r * p.ldx + c] = l;
        }
    }
}

enum { GRAM = 0, POLYNOMIAL = 1, PRODUCT = 2, LAST = 3, PART = 4 };
constexpr int BLOCK_M = 128, PAIR_M = 256, TILE_K = 64, SUM_WARPS = 16, TILED_BLOCK = 64 + 32 * SUM_WARPS;
constexpr uint32_t A_BYTES = BLOCK_M * TILE_K * 2, BOX64_BYTES = 64 * TILE_K * 2;
// One block per multiprocessor, and nothing beside it: two pairs that ask for tensor memory on the same two multiprocessors at
// the same time could each hold the right to allocate on one of them and wait for it on the other.
constexpr uint32_t TILED_SMEM = 192 * 1024 + 1024;

struct TiledArgs {
    uint32_t m, n, k_blocks;   // rows and columns of the result, runs of TILE_K values of K
    uint32_t tiles_n;          // tiles per row of tiles (PRODUCT, LAST)
    uint32_t slices;           // PART: K is cut into as many pieces (gridDim.z)
    float* part;               // PART: [slices][batch][m][ld] sums
    uint32_t ld;
};

// Barrier of the THREADS threads that put 64 columns of a tile together.
template <int THREADS> __device__ __forceinline__ void group_sync(uint32_t group) { asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(THREADS) : "memory"); }
// ... and whether `ok` holds for all of them.
template <int THREADS> __device__ __forceinline__ bool group_all(uint32_t group, bool ok)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.and.pred q, %2, %3, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)ok), "r"(1 + group), "n"(THREADS) : "memory");
    return r != 0;
}

// How many tiles of the 256 rows bi of a symmetric result reach the diagonal or lie below it.
__host__ __device__ constexpr uint32_t tiles_of_rows(uint32_t bi, uint32_t tile_n) { return (PAIR_M / tile_n) * (bi + 1); }

// A tile of 256 x TILE_N results (128 or 256) by a pair of blocks, 128 rows each.  In each block warp 0 brings in the operands' pairs by TMA; warp 1
// of the first block issues the products of both (cta_group::2: each block reads its own rows of A and half of B, so shared
// memory is read and filled at two thirds of the rate that a block on its own would need); sixteen warps sum.  The tensor cores cut
// what an addition shifts out, so a long sum in tensor memory drifts towards zero (1e-6 of a 1024-term sum, which the iteration
// multiplies: 1e-4 of the result at 4096 x 4096).  Each run of TILE_K values of K therefore starts anew in one of two or four sets
// of accumulators, the small products hi lo and lo hi first, and is added in registers, with rounding, while the next run is
// multiplied.
// The result leaves through shared memory in the operands' layout, by TMA.  Of a symmetric matrix only the 256 x 256 blocks on and
// below the diagonal are there; an operand's tile above it is its mirror image, brought in as it lies and read along the other
// axis (MN-major).
template <int MODE, int TILE_N>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(TILED_BLOCK, 1)
orth_tiled_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_mirror,
                  const __grid_constant__ CUtensorMap map_to, TiledArgs t, OrthArgs o)
{
    constexpr bool SYMMETRIC = MODE == GRAM || MODE == POLYNOMIAL || MODE == PART, MN_MAJOR = !SYMMETRIC;
    constexpr bool HALF_A = MODE == POLYNOMIAL || MODE == PRODUCT || MODE == LAST, HALF_B = MODE == POLYNOMIAL;   // operands of which only half is there
    constexpr int SETS = 512 / TILE_N;                      // of accumulators
    constexpr int OWN = TILE_N / 4, PANELS = TILE_N / 64;   // columns that a summing warp takes; runs of 64 columns
    constexpr int SHARERS = 32 * SUM_WARPS / PANELS;        // threads that put such a run together
    constexpr uint32_t B_BYTES = TILE_N / 2 * TILE_K * 2, STAGE_BYTES = 2 * (A_BYTES + B_BYTES), STAGES = TILE_N == 256 ? 3 : 4;
    static_assert(STAGES * STAGE_BYTES + 1024 == TILED_SMEM && 2 * PANELS * PANEL <= STAGES * STAGE_BYTES, "shared memory of a block");
    extern __shared__ char raw[];
    __shared__ uint64_t bars[3 * STAGES + 2 * SETS + 1];
    __shared__ uint32_t tmem_mem;
    char* base = (char*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x & 1;
    uint32_t bi = 0, bj = blockIdx.x >> 1;
    if (SYMMETRIC) {
        while (bj >= tiles_of_rows(bi, TILE_N)) bj -= tiles_of_rows(bi++, TILE_N);
    } else {
        bi = bj / t.tiles_n;
        bj -= bi * t.tiles_n;
    }
    const uint32_t row0 = bi * PAIR_M + rank * BLOCK_M, col0 = bj * TILE_N;
    uint32_t kb0 = 0, kbs = t.k_blocks;
    if (MODE == PART) {
        kb0 = (uint32_t)((uint64_t)t.k_blocks * blockIdx.z / t.slices);
        kbs = (uint32_t)((uint64_t)t.k_blocks * (blockIdx.z + 1) / t.slices) - kb0;
    }
    auto full = [&](uint32_t s) { return smem_address(&bars[s]); };                      // this block's copies have landed
    auto other = [&](uint32_t s) { return smem_address(&bars[STAGES + s]); };            // first block: the second's have
    auto empty = [&](uint32_t s) { return smem_address(&bars[2 * STAGES + s]); };
    auto summed = [&](uint32_t b) { return smem_address(&bars[3 * STAGES + b]); };       // first block: a set of accumulators is free
    auto ready = [&](uint32_t b) { return smem_address(&bars[3 * STAGES + SETS + b]); };    // ... is complete
    auto above = [&](int k0, uint32_t block) { return (uint32_t)k0 >= (block + 1) * PAIR_M; };   // columns from k0 of this block of 256 rows
    const uint32_t old_here = smem_address(&bars[3 * STAGES + 2 * SETS]);
    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < STAGES; ++s) { mbar_init(full(s), 1); mbar_init(other(s), 1); mbar_init(empty(s), 1); }
        for (int b = 0; b < SETS; ++b) { mbar_init(summed(b), 2 * SUM_WARPS); mbar_init(ready(b), 1); }
        mbar_init(old_here, 1);
        mbar_init_visible();
    }
    __syncwarp();
    if (warp == 1) tmem_alloc<2>(smem_address(&tmem_mem), SETS * TILE_N);
    tc_fence_before();
    __syncthreads();
    cluster_arrive();
    cluster_wait();                                         // both blocks' barriers are there
    tc_fence_after();
    const uint32_t tmem = tmem_mem;
    grid_dependency_wait();
    bool ok = true;
    if (warp == 0) {
        if (lane == 0) {
            asm volatile("fence.proxy.async.global;" ::: "memory");       // the first pairs were written by ordinary stores
            const uint32_t at = smem_address(base);
            const int z = 2 * (int)blockIdx.y;
            uint32_t kb = 0;
            for (; kb < kbs; ++kb) {
                const uint32_t s = kb % STAGES;
                if (kb >= STAGES && !mbar_wait(empty(s), (kb / STAGES - 1) & 1)) { ok = false; break; }
                const uint32_t to = at + s * STAGE_BYTES;
                const int k0 = (int)((kb0 + kb) * TILE_K), n0 = (int)(col0 + rank * (TILE_N / 2));
                mbar_expect(full(s), STAGE_BYTES);
                const bool mirror_a = HALF_A && above(k0, bi), mirror_b = HALF_B && above(k0, col0 / PAIR_M);
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    if (mirror_a) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) tma_load(to + p * A_BYTES + c * BOX64_BYTES, &map_mirror, (int)row0 + 64 * c, k0, z + p, full(s));
                    } else {
                        tma_load(to + p * A_BYTES, &map_a, k0, (int)row0, z + p, full(s));
                    }
                    const uint32_t to_b = to + 2 * A_BYTES + p * B_BYTES;
                    if (MN_MAJOR || mirror_b) {
#pragma unroll
                        for (int c = 0; c < TILE_N / 128; ++c) tma_load(to_b + c * BOX64_BYTES, MN_MAJOR ? &map_b : &map_mirror, n0 + 64 * c, k0, z + p, full(s));
                    } else {
                        tma_load(to_b, &map_b, k0, n0, z + p, full(s));
                    }
                }
            }
            // Whatever still comes to this block's shared memory must come before it ends: the copies in flight, and the products'
            // signals that a stage is free, which nobody else waits for at the end (a later block's barriers may lie at that place).
            for (uint32_t k = kb > STAGES ? kb - STAGES : 0; k < kb; ++k) {
                ok &= mbar_wait(full(k % STAGES), (k / STAGES) & 1);
                ok &= mbar_wait(empty(k % STAGES), (k / STAGES) & 1);
            }
            if (MODE == POLYNOMIAL) {                       // A's tile, where the result is going to be put together
                if (ok) {
                    mbar_expect(old_here, 2 * PANELS * PANEL);
                    for (int p = 0; p < 2; ++p)
                        for (int c = 0; c < PANELS; ++c) tma_load(at + (c * 2 + p) * PANEL, &map_a, (int)col0 + 64 * c, (int)row0, z + p, old_here);
                    ok = mbar_wait(old_here, 0);
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint32_t at = smem_address(base);
            for (uint32_t kb = 0; kb < kbs; ++kb) {
                const uint32_t s = kb % STAGES, b = kb % SETS;
                if ((kb >= SETS && !mbar_wait(summed(b), (kb / SETS - 1) & 1)) || !mbar_wait(full(s), (kb / STAGES) & 1) || !mbar_wait(other(s), (kb / STAGES) & 1)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t ah = at + s * STAGE_BYTES, bh = ah + 2 * A_BYTES;
                const int k0 = (int)((kb0 + kb) * TILE_K);
                const bool mn_a = HALF_A && above(k0, bi), mn_b = MN_MAJOR || (HALF_B && above(k0, col0 / PAIR_M));
                const uint32_t shape = product_shape<2>(TILE_N, mn_b, mn_a);
#pragma unroll
                for (int term = 0; term < 3; ++term) {      // hi lo, lo hi, hi hi
                    const uint32_t pa = ah + (term == 1 ? A_BYTES : 0), pb = bh + (term == 0 ? B_BYTES : 0);
#pragma unroll
                    for (int k = 0; k < TILE_K / 16; ++k) {
                        const uint64_t da = mn_a ? operand_mn_major(pa + k * 2048, BOX64_BYTES) : operand_k_major(pa + k * 32);
                        const uint64_t db = mn_b ? operand_mn_major(pb + k * 2048, BOX64_BYTES) : operand_k_major(pb + k * 32);
                        tc_product<2>(tmem + b * TILE_N, da, db, shape, term > 0 || k > 0);
                    }
                }
                tc_commit<2>(empty(s));
                tc_commit<2>(ready(b));
            }
        } else if (lane == 0) {                             // tells the first block that this block's operands are there
            for (uint32_t kb = 0; kb < kbs; ++kb) {
                const uint32_t s = kb % STAGES;
                if (!mbar_wait(full(s), (kb / STAGES) & 1)) { ok = false; break; }
                mbar_arrive_cluster(smem_of_rank(other(s), 0));
            }
        }
    } else {
        // four warps, one for each quarter of the rows, take OWN columns; group: the run of 64 columns that these belong to
        const uint32_t own_col = (warp - 2) / 4 * OWN, group = own_col / 64, quarter = (warp & 3) * 32, own_row = quarter + lane;
        float acc[OWN];
#pragma unroll
        for (int j = 0; j < OWN; ++j) acc[j] = 0.0f;
        for (uint32_t kb = 0; kb < kbs; ++kb) {
            const uint32_t b = kb % SETS;
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(ready(b), (kb / SETS) & 1));
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < OWN; c += 32) {
                float v[32];
                tmem_load32(tmem + (quarter << 16) + b * TILE_N + own_col + c, v);
#pragma unroll
                for (int j = 0; j < 32; ++j) acc[c + j] += v[j];
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(smem_of_rank(summed(b), 0));
        }
        if (MODE == POLYNOMIAL) ok = ok && mbar_wait(old_here, 0);
        ok = group_all<SHARERS>(group, ok);
        const uint32_t col = col0 + own_col;
        if (MODE == LAST || MODE == PART) {
            float* tile = (float*)base + (warp - 2) * 32 * 33;
#pragma unroll
            for (int j = 0; j < OWN; ++j) acc[j] = MODE == PART ? acc[j] * (FROM_XX * A_SCALE) : acc[j] * FROM_BX * o.scale;
#pragma unroll
            for (int c = 0; c < OWN; c += 32) {
                if (!ok || row0 + quarter >= t.m || col + c >= t.n) continue;
                const uint32_t rows = t.m - row0 - quarter, cols = t.n - col - c;
                if (MODE == PART) {
                    write_rows(t.part + ((uint64_t)blockIdx.z * gridDim.y + blockIdx.y) * t.m * t.ld, NUPS_F32, (uint64_t)(row0 + quarter) * t.ld + col + c, t.ld, rows,
                               cols, acc + c, tile);
                } else {
                    char* out = (char*)o.out + (uint64_t)blockIdx.y * o.ob * (o.type == NUPS_F32 ? 4 : 2);
                    if (!o.tall) {
                        write_rows(out, o.type, (uint64_t)(row0 + quarter) * o.os + col + c, o.os, rows, cols, acc + c, tile);
                    } else if ((uint32_t)lane < rows) {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if ((uint32_t)j < cols) write_value(out, o.type, (uint64_t)(col + c + j) * o.os + row0 + own_row, acc[c + j]);
                    }
                }
            }
        } else if (ok) {
            char* const panel = base + group * 2 * PANEL;   // hi, then lo, of the 64 columns
            const uint32_t in_panel = own_col % 64, panel_col = col0 + group * 64;
#pragma unroll
            for (int c = 0; c < OWN; c += 8) {
                char* const hi_at = panel + panel_at(own_row, in_panel + c);
                uint4 hi, lo;
                float* v = acc + c;
                if (MODE == POLYNOMIAL) {
                    hi = *(const uint4*)hi_at;
                    lo = *(const uint4*)(hi_at + PANEL);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 old = join2(((const uint32_t*)&hi)[j], ((const uint32_t*)&lo)[j]);
                        const uint32_t k = col + c + 2 * j, r = row0 + own_row;
                        v[2 * j] = o.b * old.x + o.c * (v[2 * j] * (FROM_AA * A_SCALE)) + (k == r ? o.a * A_SCALE : 0.0f);
                        v[2 * j + 1] = o.b * old.y + o.c * (v[2 * j + 1] * (FROM_AA * A_SCALE)) + (k + 1 == r ? o.a * A_SCALE : 0.0f);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] *= MODE == GRAM ? FROM_XX * A_SCALE : FROM_BX * X_SCALE;
                }
                split8(v, hi, lo);
                *(uint4*)hi_at = hi;
                *(uint4*)(hi_at + PANEL) = lo;
            }
            const bool first = (threadIdx.x - 64) % SHARERS == 0;
            const int z = 2 * (int)blockIdx.y;
            async_proxy_fence();
            group_sync<SHARERS>(group);
            if (first && row0 < t.m && panel_col < t.n) {
                tma_store(&map_to, (int)panel_col, (int)row0, z, smem_address(panel));
                tma_store(&map_to, (int)panel_col, (int)row0, z + 1, smem_address(panel + PANEL));
                tma_store_commit();
            }
            if (first) tma_store_wait_read();               // the writes are done when the grid is
        }
    }
    if (!ok) atomicCAS(&o.st->status, 0, NUPS_ETIMEOUT);
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    cluster_arrive();
    cluster_wait();                                         // nobody signals or reads the other block any more
    tc_fence_after();
    if (warp == 1) tmem_free<2>(tmem, SETS * TILE_N);
}

// A from the slices' sums, 64 x 64 values per block of 256 threads, four at a time (ld is a multiple of 8).
__global__ void __launch_bounds__(256) orth_join_kernel(const float* part, uint32_t slices, uint32_t m, uint32_t ld, __half* a)
{
    const uint32_t c0 = blockIdx.x * 64, r0 = blockIdx.y * 64, batch = gridDim.z;
    if (c0 >= (r0 / PAIR_M + 1) * PAIR_M) return;           // not computed
    grid_dependency_wait();
    const uint32_t c = c0 + (threadIdx.x & 15) * 4, ty = threadIdx.x >> 4;
    if (c >= m) return;
    float4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 2
    for (uint32_t s = 0; s < slices; ++s) {
        const float* from = part + ((uint64_t)s * batch + blockIdx.z) * m * ld + c;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t r = r0 + ty + 16 * k;
            if (r < m) v[k] = add4(v[k], __ldcg((const float4*)(from + (uint64_t)r * ld)));
        }
    }
    __half* hi = a + (uint64_t)blockIdx.z * 2 * m * ld + c;
    __half* lo = hi + (uint64_t)m * ld;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t r = r0 + ty + 16 * k;
        if (r < m) {                                        // values beyond m in a row's last run are not read by anybody
            const __half2 h0 = __floats2half2_rn(v[k].x, v[k].y), h1 = __floats2half2_rn(v[k].z, v[k].w);
            const float2 f0 = __half22float2(h0), f1 = __half22float2(h1);
            const __half2 l0 = __floats2half2_rn(v[k].x - f0.x, v[k].y - f0.y), l1 = __floats2half2_rn(v[k].z - f1.x, v[k].w - f1.y);
            *(uint2*)(hi + (uint64_t)r * ld) = make_uint2(*(const uint32_t*)&h0, *(const uint32_t*)&h1);
            *(uint2*)(lo + (uint64_t)r * ld) = make_uint2(*(const uint32_t*)&l0, *(const uint32_t*)&l1);
        }
    }
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
{
    static EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) p = nullptr;
        return (EncodeTiled)p;
    }();
    return fn;
}

// Planes of rows x cols fp16 values, `ld` apart; boxes of box_rows x box_cols, 128 bytes wide, swizzled.
nups_status plane_map(CUtensorMap* map, __half* p, uint32_t rows, uint32_t cols, uint32_t ld, uint32_t planes, uint32_t box_rows, uint32_t box_cols)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return nups_cuda_fail(cudaErrorNotSupported, "cuTensorMapEncodeTiled");
    const cuuint64_t dims[3] = {cols, rows, planes}, strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)rows * ld * 2};
    const cuuint32_t box[3] = {box_cols, box_rows, 1}, ones[3] = {1, 1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, p, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? NUPS_OK : nups_cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
}

uint64_t align_up(uint64_t x) { return (x + 255) / 256 * 256; }

bool small_form(uint32_t m, uint32_t n) { return m <= SMALL_M && n <= SMALL_N; }

uint64_t tile_pairs(uint32_t m, uint32_t n, bool symmetric, uint32_t tile_n)
{
    const uint32_t rows = (m + PAIR_M - 1) / PAIR_M;
    uint64_t tiles = 0;
    if (symmetric) for (uint32_t bi = 0; bi < rows; ++bi) tiles += tiles_of_rows(bi, tile_n);
    else tiles = (uint64_t)rows * ((n + tile_n - 1) / tile_n);
    return tiles;
}
// 256 or 128 columns per tile: what takes less time in rounds of the multiprocessors.  A run of K takes 1,550 cycles with 256
// columns (the products' own time) and 1,270 with 128, where reading the operands bounds the products: a round of the narrower
// tiles takes five sixths of the wider ones' time.
uint32_t pick_tile(const nups_store* s, uint32_t batch, uint32_t m, uint32_t n, bool symmetric)
{
    const uint64_t pairs = (uint64_t)s->sm_count / 2;
    const uint64_t wide = (tile_pairs(m, n, symmetric, 256) * batch + pairs - 1) / pairs, narrow = (tile_pairs(m, n, symmetric, 128) * batch + pairs - 1) / pairs;
    return 5 * narrow < 6 * wide ? 128 : 256;
}
// Into how many pieces K of the Gram matrix is cut where its tiles alone would leave multiprocessors idle: pieces of at least
// 512 values, one block per multiprocessor at most.
uint32_t gram_slices(const nups_store* s, uint32_t batch, uint32_t m, uint32_t n)
{
    const uint64_t fit = (uint64_t)s->sm_count / 2 / (tile_pairs(m, m, true, 256) * batch), pieces = n / 512;
    const uint64_t slices = fit < pieces ? fit : pieces;
    return slices < 2 ? 1 : slices > 8 ? 8 : (uint32_t)slices;
}

uint64_t planes_layout(const nups_store* s, uint32_t batch, uint32_t rows, uint32_t cols, char* base, Planes* p)
{
    const uint32_t m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    const uint32_t ldx = up(n, 8), lda = up(m, 8), slices = gram_slices(s, batch, m, n), parts = norm_parts(rows, cols);
    const uint64_t xb = align_up((uint64_t)batch * 2 * m * ldx * 2), ab = align_up((uint64_t)batch * 2 * m * lda * 2), sb = align_up((uint64_t)batch * parts * 8);
    if (p) *p = {{(__half*)base, (__half*)(base + xb)}, (__half*)(base + 2 * xb), (__half*)(base + 2 * xb + ab), (double*)(base + 2 * xb + 2 * ab), parts,
                 (float*)(base + 2 * xb + 2 * ab + sb), ldx, lda, slices};
    return 2 * xb + 2 * ab + sb + (slices > 1 ? (uint64_t)slices * batch * m * lda * 4 : 0);
}

#define OK_OR_RETURN(call)                     \
    do {                                       \
        const nups_status rc__ = (call);       \
        if (rc__ != NUPS_OK) return rc__;      \
    } while (0)

struct Maps { CUtensorMap rows128, rows64; };              // boxes of 128 or 64 rows and 64 columns
nups_status buffer_maps(Maps* to, __half* p, uint32_t rows, uint32_t cols, uint32_t ld, uint32_t batch)
{
    OK_OR_RETURN(plane_map(&to->rows128, p, rows, cols, ld, 2 * batch, 128, 64));
    return plane_map(&to->rows64, p, rows, cols, ld, 2 * batch, 64, 64);
}

template <int MODE, int TILE_N>
nups_status launch_tiles(nups_store* s, const Maps& a, const Maps& b, const Maps& to, const TiledArgs& t, const OrthArgs& o, unsigned batch, cudaStream_t st)
{
    constexpr bool SYMMETRIC = MODE == GRAM || MODE == POLYNOMIAL || MODE == PART;
    const unsigned tiles = (unsigned)tile_pairs(t.m, t.n, SYMMETRIC, TILE_N);
    TiledArgs u = t;
    u.tiles_n = (t.n + TILE_N - 1) / TILE_N;
    CK(nups_launch_dependent(orth_tiled_kernel<MODE, TILE_N>, dim3(2 * tiles, batch, t.slices), TILED_BLOCK, TILED_SMEM, st, a.rows128,
                             SYMMETRIC && TILE_N == 256 ? b.rows128 : b.rows64, a.rows64, to.rows128, u, o));
    LAUNCH_CHECK(s);
    return NUPS_OK;
}
template <int MODE>
nups_status launch_tiled(nups_store* s, const Maps& a, const Maps& b, const Maps& to, const TiledArgs& t, const OrthArgs& o, unsigned batch, cudaStream_t st)
{
    constexpr bool SYMMETRIC = MODE == GRAM || MODE == POLYNOMIAL || MODE == PART;
    if constexpr (MODE != PART)
        if (pick_tile(s, batch, t.m, t.n, SYMMETRIC) == 128) return launch_tiles<MODE, 128>(s, a, b, to, t, o, batch, st);
    return launch_tiles<MODE, 256>(s, a, b, to, t, o, batch, st);
}

// Large dynamic shared memory, asked for once on the store's device.
template <int MODE, int TILE_N> cudaError_t opt_in_tiled() { return cudaFuncSetAttribute(orth_tiled_kernel<MODE, TILE_N>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)TILED_SMEM); }
template <int TYPE> cudaError_t opt_in_small()
{
    const int most = (int)small_smem(SMALL_M, SMALL_N);
    const cudaError_t e = cudaFuncSetAttribute(orthogonalize_small_kernel<TYPE, 256>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(orthogonalize_small_kernel<TYPE, 512>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
}
template <int TYPE> nups_status launch_small(nups_store* s, const OrthArgs& o, uint32_t batch, cudaStream_t st)
{
    const unsigned block = o.n > 64 ? 512 : 256;            // o.m <= o.n
    CK(nups_launch_dependent(block == 512 ? orthogonalize_small_kernel<TYPE, 512> : orthogonalize_small_kernel<TYPE, 256>, dim3(batch), block, small_smem(o.m, o.n), st, o));
    LAUNCH_CHECK(s);
    return NUPS_OK;
}
nups_status opt_in(nups_store* s)
{
    if (s->orth_smem_opted) return NUPS_OK;
    CK(opt_in_small<NUPS_F32>());
    CK(opt_in_small<NUPS_F16>());
    CK(opt_in_small<NUPS_BF16>());
    CK((opt_in_tiled<GRAM, 128>()));
    CK((opt_in_tiled<GRAM, 256>()));
    CK((opt_in_tiled<POLYNOMIAL, 128>()));
    CK((opt_in_tiled<POLYNOMIAL, 256>()));
    CK((opt_in_tiled<PRODUCT, 128>()));
    CK((opt_in_tiled<PRODUCT, 256>()));
    CK((opt_in_tiled<LAST, 128>()));
    CK((opt_in_tiled<LAST, 256>()));
    CK((opt_in_tiled<PART, 256>()));
    s->orth_smem_opted = true;
    return NUPS_OK;
}

nups_status launch_large(nups_store* s, const OrthArgs& o, uint32_t batch, char* scratch, cudaStream_t st)
{
    Planes p;
    planes_layout(s, batch, o.rows, o.cols, scratch, &p);
    Maps x[2], a, b;
    for (int i = 0; i < 2; ++i) OK_OR_RETURN(buffer_maps(&x[i], p.x[i], o.m, o.n, p.ldx, batch));
    OK_OR_RETURN(buffer_maps(&a, p.a, o.m, o.m, p.lda, batch));
    OK_OR_RETURN(buffer_maps(&b, p.b, o.m, o.m, p.lda, batch));
    nups_launch_dependent(orth_squares_kernel, dim3(p.parts, batch), 256, 0, st, o, p.sums);
    LAUNCH_CHECK(s);
    nups_launch_dependent(orth_split_kernel, dim3((o.n + 63) / 64, (o.m + 63) / 64, batch), 256, 0, st, o, p);
    LAUNCH_CHECK(s);
    const TiledArgs gram = {o.m, o.m, (o.n + TILE_K - 1) / TILE_K, 0, p.slices, p.part, p.lda};
    const TiledArgs polynomial = {o.m, o.m, (o.m + TILE_K - 1) / TILE_K, 0, 1, nullptr, p.lda};
    const TiledArgs product = {o.m, o.n, (o.m + TILE_K - 1) / TILE_K, 0, 1, nullptr, p.ldx};
    for (uint32_t step = 0; step < o.steps; ++step) {
        const Maps &from = x[step & 1], &to = x[1 - (step & 1)];
        if (p.slices > 1) {
            OK_OR_RETURN(launch_tiled<PART>(s, from, from, a, gram, o, batch, st));
            nups_launch_dependent(orth_join_kernel, dim3((o.m + 63) / 64, (o.m + 63) / 64, batch), 256, 0, st, (const float*)p.part, p.slices, o.m, p.lda, p.a);
            LAUNCH_CHECK(s);
        } else {
            OK_OR_RETURN(launch_tiled<GRAM>(s, from, from, a, gram, o, batch, st));
        }
        OK_OR_RETURN(launch_tiled<POLYNOMIAL>(s, a, a, b, polynomial, o, batch, st));
        if (step + 1 < o.steps) OK_OR_RETURN(launch_tiled<PRODUCT>(s, b, from, to, product, o, batch, st));
        else OK_OR_RETURN(launch_tiled<LAST>(s, b, from, to, product, o, batch, st));
    }
    return NUPS_OK;
}

// Does the iteration stay within the range of the pairs for singular values in [0, 1]?  p(s) = s (a + b s^2 + c s^4) takes [0, top] to an
// interval that begins at 0, so a step's largest value is that of |p| at top or where p' = a + 3 b u + 5 c u^2, u = s^2, is zero,
// and the factor's is at 0, at top or at u = -b / 2c.  Exact for all singular values; samples of them missed the few that run away.
bool coefficients_fit(const float* h, uint32_t steps)
{
    const double a = h[0], b = h[1], c = h[2];
    if (!isfinite(a) || !isfinite(b) || !isfinite(c)) return false;
    auto factor = [&](double u) { return fabs(a + u * (b + u * c)); };
    // zeros of q(u) = a + 3 b u + 5 c u^2, by the form that does not cancel; none: infinity or NaN, which the bounds below leave out
    const double root = sqrt(9 * b * b - 20 * a * c), q = -1.5 * b - copysign(0.5 * root, b);
    const double turns[2] = {q / (5 * c), a / q}, bend = -b / (2 * c);
    double top = 1.0;                                       // largest square of a singular value
    for (uint32_t k = 0; k < steps; ++k) {
        double f = fmax(factor(0.0), factor(top)), s = sqrt(top) * factor(top);
        if (bend > 0 && bend < top) f = fmax(f, factor(bend));
        for (double u : turns)
            if (u > 0 && u < top) s = fmax(s, sqrt(u) * factor(u));
        if (!(f <= 7.5) || !(s <= 2.5)) return false;
        top = s * s;
    }
    return true;
}

bool matrix_fits(uint64_t stride, uint64_t batch_stride, uint32_t batch, uint32_t rows, uint32_t cols)
{
    if (stride >= (1ull << 40) || batch_stride >= (1ull << 50)) return false;
    const uint64_t span = (uint64_t)(rows - 1) * (rows > 1 ? stride : 0) + cols;
    return (rows <= 1 || stride >= cols) && (batch <= 1 || batch_stride >= span);
}

}  // namespace

extern "C" nups_status nups_orthogonalize_scratch(nups_store* s, uint32_t batch, uint32_t rows, uint32_t cols, uint64_t* h_bytes_out)
{
    if (!s || !h_bytes_out || batch > 65535 || rows < 1 || cols < 1 || rows > NUPS_ORTHOGONALIZE_MAX_SIZE || cols > NUPS_ORTHOGONALIZE_MAX_SIZE) return NUPS_EINVAL;
    const uint32_t m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    *h_bytes_out = small_form(m, n) || batch == 0 ? 0 : planes_layout(s, batch, rows, cols, nullptr, nullptr);
    return NUPS_OK;
}

extern "C" nups_status nups_orthogonalize(nups_store* s, const void* d_update, int type, uint64_t stride, uint64_t batch_stride, uint32_t batch,
                                          uint32_t rows, uint32_t cols, uint32_t steps, const float* h_coefficients, float eps, float scale,
                                          void* d_out, uint64_t out_stride, uint64_t out_batch_stride, void* d_scratch, uint64_t scratch_bytes,
                                          void* stream)
{
    uint64_t bytes = 0;
    if (!s || (type != NUPS_F32 && type != NUPS_F16 && type != NUPS_BF16) || nups_orthogonalize_scratch(s, batch, rows, cols, &bytes) != NUPS_OK) return NUPS_EINVAL;
    if (steps < 1 || steps > NUPS_ORTHOGONALIZE_MAX_STEPS || !h_coefficients || !coefficients_fit(h_coefficients, steps) || !(eps > 0) || !isfinite(eps) || !isfinite(scale))
        return NUPS_EINVAL;
    if (!matrix_fits(stride, batch_stride, batch, rows, cols) || !matrix_fits(out_stride, out_batch_stride, batch, rows, cols)) return NUPS_EINVAL;
    if ((batch && (!d_update || !d_out)) || !suits(type_bytes(type), d_update, d_out)) return NUPS_EINVAL;
    if (batch && bytes && (!d_scratch || scratch_bytes < bytes || ((uintptr_t)d_scratch & 255))) return NUPS_EINVAL;
    nups_status rc = on_own_device(s);
    if (rc != NUPS_OK || batch == 0) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    const bool tall = rows > cols;
    const OrthArgs o = {d_update, d_out, stride, batch_stride, out_stride, out_batch_stride, rows, cols, tall ? cols : rows, tall ? rows : cols, steps, type, tall,
                        h_coefficients[0], h_coefficients[1], h_coefficients[2], eps, scale, s->st};
    rc = opt_in(s);
    if (rc != NUPS_OK) return rc;
    if (small_form(o.m, o.n))
        return type == NUPS_F32 ? launch_small<NUPS_F32>(s, o, batch, st) : type == NUPS_F16 ? launch_small<NUPS_F16>(s, o, batch, st) : launch_small<NUPS_BF16>(s, o, batch, st);
    return launch_large(s, o, batch, (char*)d_scratch, st);
}
