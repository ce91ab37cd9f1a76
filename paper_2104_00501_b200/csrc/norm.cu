// Layer norm of dense rows and of pulled rows, and its backward pass.
//
// y = (x - mean) rstd w + b is bound by memory: x is read once, y written once, some eight operations a value.  A row is held in
// the registers of a team of TPR threads (CH chunks of VEC values each), so the variance is taken about the mean in a second pass
// over registers, not as a difference of sums; w and b stay in registers while a team walks its rows.  A team works on ROWS rows
// at a time: their loads are in flight together and their reductions overlap.  Teams of up to 32 threads reduce by shuffles; a
// block that is one team merges its warps' (sum, sum of squares about the warp's own mean) with one barrier per ROWS rows (Chan's
// formula for the variance of a union).
#include <atomic>

#include "nups_tcgen05.cuh"
#include "nups_types.cuh"

namespace {

struct NormArgs {
    const void* x;
    uint64_t xs;
    void* y;
    uint64_t ys;
    const void *w, *b;
    void *mean, *rstd;
    uint64_t n;
    uint32_t len;
    int y_type, w_type, w_vec;
    double eps;
    const uint32_t* keys;      // pull_norm: rows come from the store
    void* rows;
    DevStat* st;
};

// Values that thread t of a team of TPR holds: chunk c covers VEC values from (c * TPR + t) * VEC.
template <int TPR, int VEC> __device__ __forceinline__ uint32_t value_at(int c, int t) { return (uint32_t)(c * TPR + t) * VEC; }

// EPT parameters of a thread (weight or bias), widened; `fill` where there are none.
template <class X, class A, int VEC, int TPR, int CH>
__device__ __forceinline__ void load_params(const void* p, int type, int vec, uint32_t len, int t, A fill, A (&out)[CH][VEC])
{
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const uint32_t at = value_at<TPR, VEC>(c, t);
#pragma unroll
        for (int j = 0; j < VEC; ++j) out[c][j] = fill;
        if (p && at < len) {
            if (sizeof(X) == 2 && type == NUPS_F32) {
                if (vec) unpack<A>(load_pack<float, VEC>((const float*)p + at), out[c]);
                else
#pragma unroll
                    for (int j = 0; j < VEC; ++j) out[c][j] = widen<A>(((const float*)p)[at + j]);
            } else {
                if (vec) unpack<A>(load_pack<X, VEC>((const X*)p + at), out[c]);
                else
#pragma unroll
                    for (int j = 0; j < VEC; ++j) out[c][j] = widen<A>(((const X*)p)[at + j]);
            }
        }
    }
}

// The VEC parameters from value `at` on.
template <class X, class A, int VEC>
__device__ __forceinline__ void load_params_at(const void* p, int type, int vec, uint32_t at, A fill, A (&out)[1][VEC])
{
    const size_t size = sizeof(X) == 2 && type == NUPS_F32 ? 4 : sizeof(X);
    load_params<X, A, VEC, 1, 1>(p ? (const char*)p + (size_t)at * size : nullptr, type, vec, VEC, 0, fill, out);
}

// One chunk of an output whose type is X, or for fp32 X also a 16-bit type.
template <class X, class A, int VEC>
__device__ __forceinline__ void store_chunk(void* p, int type, uint64_t at, const A* v)
{
    if constexpr (sizeof(X) == 4) {
        if (type == NUPS_BF16) return store_values<__nv_bfloat16, VEC>((__nv_bfloat16*)p + at, v);
        if (type == NUPS_F16) return store_values<__half, VEC>((__half*)p + at, v);
    }
    store_values<X, VEC>((X*)p + at, v);
}
template <class X, class A, int VEC>
__device__ __forceinline__ void load_chunk(const void* p, int type, uint64_t at, A* v)
{
    if constexpr (sizeof(X) == 4) {
        if (type == NUPS_BF16) return unpack<A>(load_pack<__nv_bfloat16, VEC>((const __nv_bfloat16*)p + at), v);
        if (type == NUPS_F16) return unpack<A>(load_pack<__half, VEC>((const __half*)p + at), v);
    }
    unpack<A>(load_pack<X, VEC>((const X*)p + at), v);
}

template <int W, class A> __device__ __forceinline__ A team_sum(A x)
{
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

template <class A> __device__ __forceinline__ A inv_sqrt(A x);
template <> __device__ __forceinline__ float inv_sqrt<float>(float x) { return 1.0f / sqrtf(x); }
template <> __device__ __forceinline__ double inv_sqrt<double>(double x) { return 1.0 / sqrt(x); }

template <class X> struct Acc { typedef float type; };
template <> struct Acc<double> { typedef double type; };

__host__ __device__ constexpr int team_block(int tpr) { return tpr > 32 ? tpr : 256; }

// ---------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------
// Mean and reciprocal deviation of ROWS rows; x(k, c, v) gives the thread's chunk c of row k (zero beyond len), sync() is the barrier
// of a block that is one team.
template <class A, int VEC, int TPR, int CH, int ROWS, class Get, class Sync>
__device__ __forceinline__ void row_stats(Get x, Sync sync, uint32_t len, A eps, int t, int turn, A* shared, A (&mean)[ROWS], A (&rstd)[ROWS])
{
    constexpr int WARPS = TPR / 32, LANES = TPR < 32 ? TPR : 32;
    A sum[ROWS], sq[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        A acc[2] = {0, 0};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            A v[VEC];
            x(k, c, v);
            sum_run<VEC>(acc, v);
        }
        sum[k] = acc[0] + acc[1];
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) sum[k] = team_sum<LANES>(sum[k]);
    uint32_t held = len;                                    // values of the row that the warp holds; the squares are taken about their mean
    if (TPR > 32) {
        held = 0;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const uint32_t at = value_at<TPR, VEC>(c, t & ~31);
            held += at < len ? min((uint32_t)(32 * VEC), len - at) : 0u;
        }
    }
    const A inv_held = held ? (A)1 / (A)held : (A)0;
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        mean[k] = TPR > 32 ? sum[k] * inv_held : sum[k] / (A)len;
        const A minus = -mean[k];
        A acc[2] = {0, 0};
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (value_at<TPR, VEC>(c, t) < len) {
                A v[VEC];
                x(k, c, v);
                run_add<VEC, true>(v, v, &minus);
                sum_run_of_products<VEC>(acc, v, v);
            }
        sq[k] = acc[0] + acc[1];
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) sq[k] = team_sum<LANES>(sq[k]);
    if (TPR > 32) {
        // lanes [k WARPS, (k + 1) WARPS) take row k's warps; 32 / WARPS rows at a time
        constexpr int AT_ONCE = 32 / (WARPS > 0 ? WARPS : 1) < ROWS ? 32 / (WARPS > 0 ? WARPS : 1) : ROWS;
        A* st = shared + (turn & 1) * (2 * ROWS + 1) * WARPS;             // two sets: the next rows' is written while this one is read
        const int warp = t >> 5, lane = t & 31;
        if (lane == 0) {
#pragma unroll
            for (int k = 0; k < ROWS; ++k) { st[k * WARPS + warp] = sum[k]; st[(ROWS + k) * WARPS + warp] = sq[k]; }
            st[2 * ROWS * WARPS + warp] = (A)held;
        }
        sync();
#pragma unroll
        for (int k0 = 0; k0 < ROWS; k0 += AT_ONCE) {
            const int k = k0 + (lane / (WARPS > 0 ? WARPS : 1)) % AT_ONCE, w = lane % (WARPS > 0 ? WARPS : 1);
            const A s = st[k * WARPS + w], q = st[(ROWS + k) * WARPS + w], h = st[2 * ROWS * WARPS + w];
            const A m = team_sum<WARPS>(s) / (A)len;
            const A d = h > 0 ? s / h - m : (A)0;
            const A r = inv_sqrt<A>(team_sum<WARPS>(q + h * d * d) / (A)len + eps);
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                mean[k0 + i] = __shfl_sync(0xFFFFFFFFu, m, i * WARPS);
                rstd[k0 + i] = __shfl_sync(0xFFFFFFFFu, r, i * WARPS);
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) rstd[k] = inv_sqrt<A>(sq[k] / (A)len + eps);
    }
}

template <class X, int VEC, int TPR, int CH, int ROWS, bool KEYED>
__global__ void __launch_bounds__(team_block(TPR)) norm_kernel(NormArgs a, View v)
{
    typedef typename Acc<X>::type A;
    constexpr int TEAMS = team_block(TPR) / TPR;
    constexpr bool HOLD = TPR < 1024;                       // 64 registers a thread leave no room for the parameters
    __shared__ A shared[TPR > 32 ? 2 * (2 * ROWS + 1) * (TPR / 32) : 1];
    grid_dependency_wait();
    const int t = threadIdx.x % TPR, team = threadIdx.x / TPR;
    A w[CH][VEC], b[CH][VEC];
    if (HOLD) {
        load_params<X, A, VEC, TPR, CH>(a.w, a.w_type, a.w_vec, a.len, t, (A)1, w);
        load_params<X, A, VEC, TPR, CH>(a.b, a.w_type, a.w_vec, a.len, t, (A)0, b);
    }
    int turn = 0;
    // pull_norm: the lookups run ahead of the rows, the key two turns, the word that tells whether it is replicated one
    const uint64_t step = (uint64_t)gridDim.x * (TEAMS * ROWS);
    uint32_t key_a[ROWS], key_b[ROWS], bits_a[ROWS];
    auto key_of = [&](uint64_t row) { return row < a.n ? __ldg(a.keys + row) : 0u; };
    auto bits_of = [&](uint32_t key) { return v.H != 0 && key < v.num_keys ? __ldg(v.hot_bits + (key >> 5)) : 0u; };
    if constexpr (KEYED)
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const uint64_t row = (uint64_t)blockIdx.x * (TEAMS * ROWS) + k * TEAMS + team;
            key_a[k] = key_of(row);
            key_b[k] = key_of(row + step);
            bits_a[k] = bits_of(key_a[k]);
        }
    for (uint64_t base = (uint64_t)blockIdx.x * (TEAMS * ROWS); base < a.n; base += step, ++turn) {
        Pack<X, VEC> x[ROWS][CH];
        const X* src[ROWS];
        const X* pend[ROWS];
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const uint64_t row = base + k * TEAMS + team;
            src[k] = pend[k] = nullptr;
            if constexpr (KEYED) {
                const uint32_t key = key_a[k], bits = bits_a[k];
                key_a[k] = key_b[k];
                bits_a[k] = bits_of(key_a[k]);
                key_b[k] = key_of(row + 2 * step);
                if (row < a.n) {
                    if (key < v.num_keys) {
                        src[k] = (const X*)v.val + (uint64_t)key * a.len;
                        if ((bits >> (key & 31)) & 1u) {
                            const uint32_t slot = (uint32_t)__ldg(v.slot_of + key);
                            pend[k] = (const X*)v.dval + ((uint64_t)worker_of_item(row, a.n, v.R) * v.Hcap + slot) * a.len;
                        }
                        if (v.count && t == 0) {
                            atomicAdd(v.cnt + key, 1ull);
                            atomicAdd(pend[k] ? &v.st->hot_hits : &v.st->cold_hits, 1ull);
                        }
                    } else if (t == 0) {
                        flag_bad_key(v);
                    }
                }
            } else if (row < a.n) {
                src[k] = (const X*)a.x + row * a.xs;
            }
        }
#pragma unroll
        for (int k = 0; k < ROWS; ++k)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const uint32_t at = value_at<TPR, VEC>(c, t);
                if (src[k] && at < a.len) x[k][c] = load_pack<X, VEC>(src[k] + at);
                else x[k][c] = Pack<X, VEC>{};
            }
        if constexpr (KEYED) {
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                const uint64_t row = base + k * TEAMS + team;
                if (pend[k])
#pragma unroll
                    for (int c = 0; c < CH; ++c) {
                        const uint32_t at = value_at<TPR, VEC>(c, t);
                        if (at < a.len) {
                            const Pack<X, VEC> d = load_pack<X, VEC>(pend[k] + at);
#pragma unroll
                            for (int j = 0; j < VEC; ++j) x[k][c].v[j] += d.v[j];
                        }
                    }
                if (a.rows && row < a.n)
#pragma unroll
                    for (int c = 0; c < CH; ++c) {
                        const uint32_t at = value_at<TPR, VEC>(c, t);
                        if (at < a.len) store_pack<X, VEC>((X*)a.rows + row * a.len + at, x[k][c]);
                    }
            }
        }
        A mean[ROWS], rstd[ROWS];
        row_stats<A, VEC, TPR, CH, ROWS>([&](int k, int c, A* to) { unpack<A>(x[k][c], to); }, [] { __syncthreads(); }, a.len, (A)a.eps, t, turn, shared, mean, rstd);
        if (t == 0) {
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                const uint64_t row = base + k * TEAMS + team;
                if (row < a.n) {
                    if (a.mean) ((A*)a.mean)[row] = mean[k];
                    if (a.rstd) ((A*)a.rstd)[row] = rstd[k];
                }
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const uint32_t at = value_at<TPR, VEC>(c, t);
            if (at < a.len) {
                A wc[1][VEC], bc[1][VEC];
                if (!HOLD) {
                    load_params_at<X, A, VEC>(a.w, a.w_type, a.w_vec, at, (A)1, wc);
                    load_params_at<X, A, VEC>(a.b, a.w_type, a.w_vec, at, (A)0, bc);
                }
#pragma unroll
                for (int k = 0; k < ROWS; ++k) {
                    const uint64_t row = base + k * TEAMS + team;
                    const A minus = -mean[k];
                    A y[VEC];
                    unpack<A>(x[k][c], y);
                    run_add<VEC, true>(y, y, &minus);       // x - mean first: x rstd - mean rstd would leave the roundings of both products
                    run_scale<VEC>(y, y, rstd[k]);
                    run_fma<VEC, false, false, false>(y, y, HOLD ? w[c] : wc[0], HOLD ? b[c] : bc[0]);
                    if (row < a.n) store_chunk<X, A, VEC>(a.y, a.y_type, row * a.ys + at, y);
                }
            }
        }
    }
}

// Rows of 1 KB and more: the rows come into a ring of STAGES groups of ROWS rows in shared memory by bulk copies, a group or two ahead
// of the arithmetic, which reads them there three times; what is in flight takes no registers and does not stop at the block's barrier.
// (16,384 rows of 4096 bf16: 55 us with the rows in registers, two blocks of 256 threads per multiprocessor.)
template <class X, int TPR, int CH, int ROWS, int STAGES>
__global__ void __launch_bounds__(TPR) norm_ring_kernel(NormArgs a)
{
    typedef typename Acc<X>::type A;
    constexpr int VEC = 16 / sizeof(X);
    constexpr bool HOLD = CH * VEC * TPR * sizeof(A) <= 32768;            // up to 32 registers of parameters where a thread may have them
    extern __shared__ __align__(128) char ring[];
    __shared__ A shared[2 * (2 * ROWS + 1) * (TPR / 32)];
    __shared__ uint64_t bars[STAGES];
    const int t = threadIdx.x;
    const uint32_t bytes = a.len * sizeof(X), stage_bytes = bytes * ROWS;
    const uint64_t step = (uint64_t)gridDim.x * ROWS, first = (uint64_t)blockIdx.x * ROWS;
    auto bar = [&](uint32_t s) { return smem_address(&bars[s]); };
    if (t == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(bar(s), 1);
        mbar_init_visible();
    }
    grid_dependency_wait();
    auto issue = [&](uint32_t i) {                          // the block's group i; one thread
        const uint64_t base = first + i * step;
        if (base >= a.n) return;
        const uint32_t rows = (uint32_t)min((uint64_t)ROWS, a.n - base), s = i % STAGES, to = smem_address(ring) + s * stage_bytes;
        mbar_expect(bar(s), rows * bytes);
        if (a.xs == a.len) bulk_load(to, (const X*)a.x + base * a.xs, rows * bytes, bar(s));
        else
            for (uint32_t k = 0; k < rows; ++k) bulk_load(to + k * bytes, (const X*)a.x + (base + k) * a.xs, bytes, bar(s));
    };
    if (t == 0)
        for (uint32_t i = 0; i + 1 < STAGES; ++i) issue(i);
    A w[CH][VEC], b[CH][VEC];
    if (HOLD) {
        load_params<X, A, VEC, TPR, CH>(a.w, a.w_type, a.w_vec, a.len, t, (A)1, w);
        load_params<X, A, VEC, TPR, CH>(a.b, a.w_type, a.w_vec, a.len, t, (A)0, b);
    }
    __syncthreads();                                        // the barriers are there
    uint32_t i = 0;
    bool ok = true;
    for (uint64_t base = first; base < a.n; base += step, ++i) {
        const uint32_t s = i % STAGES;
        const X* x = (const X*)(ring + s * stage_bytes);
        ok = mbar_wait(bar(s), (i / STAGES) & 1);
        bool stop = false;
        auto get = [&](int k, int c, A* to) {
            const uint32_t at = value_at<TPR, VEC>(c, t);
            if (at < a.len) unpack<A>(load_pack<X, VEC>(x + k * a.len + at), to);
            else
#pragma unroll
                for (int j = 0; j < VEC; ++j) to[j] = 0;
        };
        A mean[ROWS], rstd[ROWS];
        row_stats<A, VEC, TPR, CH, ROWS>(get, [&] { stop = __syncthreads_or(!ok); }, a.len, (A)a.eps, t, (int)i, shared, mean, rstd);
        if (stop) { ok = false; break; }
        if (t == 0) {                                       // every thread is done with the group before this one
            issue(i + STAGES - 1);
#pragma unroll
            for (int k = 0; k < ROWS; ++k)
                if (base + k < a.n) {
                    if (a.mean) ((A*)a.mean)[base + k] = mean[k];
                    if (a.rstd) ((A*)a.rstd)[base + k] = rstd[k];
                }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const uint32_t at = value_at<TPR, VEC>(c, t);
            if (at < a.len) {
                A wc[1][VEC], bc[1][VEC];
                if (!HOLD) {
                    load_params_at<X, A, VEC>(a.w, a.w_type, a.w_vec, at, (A)1, wc);
                    load_params_at<X, A, VEC>(a.b, a.w_type, a.w_vec, at, (A)0, bc);
                }
#pragma unroll
                for (int k = 0; k < ROWS; ++k) {
                    const A minus = -mean[k];
                    A y[VEC];
                    get(k, c, y);
                    run_add<VEC, true>(y, y, &minus);       // as in norm_kernel
                    run_scale<VEC>(y, y, rstd[k]);
                    run_fma<VEC, false, false, false>(y, y, HOLD ? w[c] : wc[0], HOLD ? b[c] : bc[0]);
                    if (base + k < a.n) store_chunk<X, A, VEC>(a.y, a.y_type, (base + k) * a.ys + at, y);
                }
            }
        }
    }
    if (!ok) {                                              // a copy did not come: say so, and leave none in flight
        atomicCAS(&a.st->status, 0, NUPS_ETIMEOUT);
        if (t == 0)
            for (uint32_t k = i + 1; k < i + STAGES - 1; ++k)
                if (first + k * step < a.n) mbar_wait(bar(k % STAGES), (k / STAGES) & 1);
    }
}

// Sum over a block of 1024 threads, given to all of them.
template <class A> __device__ __forceinline__ A block_sum(A x, A* shared)
{
    x = team_sum<32>(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = x;
    __syncthreads();
    return team_sum<32>(shared[threadIdx.x & 31]);
}

// Rows too long for registers: a block per row reads it three times, mostly from L2.  A thread adds up to 2^18 values one after the other:
// runs of VEC in A, the runs in fp64 (in fp32 the mean of 2^25 values of 0.1 was off by 2.6e-4 of itself, and y was 0.008 instead of 0).
// 64 rows of 2^20 floats 293 us, 2,000 rows of 33,000 bf16 105 us.
template <class X, int VEC, bool KEYED>
__global__ void __launch_bounds__(1024) norm_long_kernel(NormArgs a, View v)
{
    typedef typename Acc<X>::type A;
    __shared__ double shared[32];
    grid_dependency_wait();
    for (uint64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const X* src = nullptr;
        const X* pend = nullptr;
        if (KEYED) {
            const uint32_t key = __ldg(a.keys + row);
            if (key < v.num_keys) {
                src = (const X*)v.val + (uint64_t)key * a.len;
                if (key_is_hot(v, key)) pend = (const X*)v.dval + ((uint64_t)worker_of_item(row, a.n, v.R) * v.Hcap + (uint32_t)__ldg(v.slot_of + key)) * a.len;
                if (v.count && threadIdx.x == 0) {
                    atomicAdd(v.cnt + key, 1ull);
                    atomicAdd(pend ? &v.st->hot_hits : &v.st->cold_hits, 1ull);
                }
            } else if (threadIdx.x == 0) {
                flag_bad_key(v);
            }
        } else {
            src = (const X*)a.x + row * a.xs;
        }
        auto read = [&](uint32_t at, A* x) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[j] = 0;
            if (src) unpack<A>(load_pack<X, VEC>(src + at), x);
            if (KEYED && pend) {
                A d[VEC];
                unpack<A>(load_pack<X, VEC>(pend + at), d);
#pragma unroll
                for (int j = 0; j < VEC; ++j) x[j] += d[j];
            }
        };
        double sum = 0, sq = 0;
        for (uint32_t at = threadIdx.x * VEC; at < a.len; at += 1024 * VEC) {
            A x[VEC], run = 0;
            read(at, x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) run += x[j];
            sum += (double)run;
        }
        const A mean = (A)(block_sum(sum, shared) / (double)a.len);
        for (uint32_t at = threadIdx.x * VEC; at < a.len; at += 1024 * VEC) {
            A x[VEC], run = 0;
            read(at, x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) run += (x[j] - mean) * (x[j] - mean);
            sq += (double)run;
        }
        const A rstd = inv_sqrt<A>((A)(block_sum(sq, shared) / (double)a.len) + (A)a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) ((A*)a.mean)[row] = mean;
            if (a.rstd) ((A*)a.rstd)[row] = rstd;
        }
        for (uint32_t at = threadIdx.x * VEC; at < a.len; at += 1024 * VEC) {
            A x[VEC], w[1][VEC], b[1][VEC], y[VEC];
            read(at, x);
            if (KEYED && a.rows) store_values<X, VEC>((X*)a.rows + row * a.len + at, x);
            load_params_at<X, A, VEC>(a.w, a.w_type, a.w_vec, at, (A)1, w);
            load_params_at<X, A, VEC>(a.b, a.w_type, a.w_vec, at, (A)0, b);
#pragma unroll
            for (int j = 0; j < VEC; ++j) y[j] = (x[j] - mean) * rstd * w[0][j] + b[0][j];
            store_chunk<X, A, VEC>(a.y, a.y_type, row * a.ys + at, y);
        }
    }
}

// Blocks of a kernel that a multiprocessor holds at once: grids of whole waves, as a team loads its parameters once per block.
template <class... KArgs> unsigned resident_blocks(void (*kernel)(KArgs...), int block)
{
    int n = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, block, 0) != cudaSuccess) cudaGetLastError();
    return n > 0 ? (unsigned)n : 1u;
}

// The same with dynamic shared memory.  `largest`, what the kernel's longest rows need, is asked for once per device: the limit is the
// kernel's, not the call's, and another thread's call with shorter rows must not lower it between this call's asking and its launch.
// The size of this call decides how many blocks fit; the last answer is remembered (device, size, blocks: one word, so that
// threads see all of one answer), as the query takes half a microsecond.
struct RingLimits { std::atomic<uint64_t> asked{0}, last{0}; };
template <class... KArgs> unsigned ring_blocks(RingLimits& known, int device, void (*kernel)(KArgs...), int block, size_t largest, size_t smem)
{
    if (device >= 64 || !(known.asked.load(std::memory_order_acquire) >> device & 1)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)largest) != cudaSuccess) return 0;
        if (device < 64) known.asked.fetch_or(1ull << device, std::memory_order_release);
    }
    const uint64_t key = ((uint64_t)(device + 1) << 48) | ((uint64_t)smem << 16), seen = known.last.load(std::memory_order_relaxed);
    if ((seen & ~0xFFFFull) == key) return (unsigned)(seen & 0xFFFF);
    int n = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, block, smem) != cudaSuccess || n < 1) return 0;
    known.last.store(key | (uint64_t)n, std::memory_order_relaxed);
    return (unsigned)n;
}

// Chunks per thread and threads per row by the number of chunks of a row; ROWS so that a thread has some 64 bytes in flight.
template <class X, int VEC, bool KEYED>
nups_status launch_norm(nups_store* s, const NormArgs& a, const View& v, cudaStream_t st)
{
    const uint32_t chunks = (a.len + VEC - 1) / VEC;
#define NUPS_RING(TPR_, CH_, ROWS_, STAGES_)                                                                                               \
    {                                                                                                                                      \
        constexpr size_t largest = (size_t)STAGES_ * ROWS_ * TPR_ * CH_ * 16;                                                              \
        const size_t smem = (size_t)STAGES_ * ROWS_ * a.len * sizeof(X);                                                                   \
        static RingLimits known;                                                                                                           \
        const unsigned resident = ring_blocks(known, s->device, norm_ring_kernel<X, TPR_, CH_, ROWS_, STAGES_>, TPR_, largest, smem);      \
        if (!resident) return nups_cuda_fail(cudaGetLastError(), "norm_ring_kernel");                                                      \
        const unsigned grid = grid_for(a.n, ROWS_, (unsigned)s->sm_count * resident);                                                      \
        nups_launch_dependent(norm_ring_kernel<X, TPR_, CH_, ROWS_, STAGES_>, grid, TPR_, smem, st, a);                                    \
        LAUNCH_CHECK(s);                                                                                                                   \
        return NUPS_OK;                                                                                                                    \
    }
    if constexpr (VEC * sizeof(X) == 16 && !KEYED) {
        if (chunks > 64 && a.n > (uint64_t)s->sm_count) {   // fewer rows: every block has one group, nothing to run ahead of
            if (chunks <= 128) NUPS_RING(128, 1, 4, 3)
            if (chunks <= 256) NUPS_RING(128, 2, 4, 3)
            if (chunks <= 512) NUPS_RING(256, 2, 4, 2)
            if (chunks <= 1024) NUPS_RING(512, 2, 2, 3)
            if (chunks <= 2048) NUPS_RING(1024, 2, 2, 3)
            if (chunks <= 4096) NUPS_RING(1024, 4, 1, 3)
        }
    }
#undef NUPS_RING
#define NUPS_NORM(TPR_, CH_, ROWS_)                                                                                                        \
    {                                                                                                                                      \
        constexpr int PER_BLOCK = team_block(TPR_) / TPR_ * ROWS_;                                                                         \
        static const unsigned resident = resident_blocks(norm_kernel<X, VEC, TPR_, CH_, ROWS_, KEYED>, team_block(TPR_));                  \
        const unsigned grid = grid_for(a.n, PER_BLOCK, (unsigned)s->sm_count * resident);                                                  \
        nups_launch_dependent(norm_kernel<X, VEC, TPR_, CH_, ROWS_, KEYED>, grid, team_block(TPR_), 0, st, a, v);                          \
    }
    if constexpr (VEC * sizeof(X) == 16) {
        // short rows: several teams to a warp with a few chunks per lane, one row each (1M pulled rows of 128 floats, the kernel by
        // itself: 205 us with 8 lanes of 4 chunks, 209 with 16 of 2, two rows each, 278 with 32 of 1, four rows each; the lookups'
        // running ahead took the first to 197.  Among other calls it takes 208.)
        if (chunks <= 4) NUPS_NORM(4, 1, 2)
        else if (chunks <= 8) NUPS_NORM(4, 2, 1)
        else if (chunks <= 16) NUPS_NORM((VEC <= 4 ? 4 : 8), (VEC <= 4 ? 4 : 2), 1)
        else if (chunks <= 32) NUPS_NORM((VEC <= 4 ? 8 : 16), (VEC <= 4 ? 4 : 2), 1)
        else if (chunks <= 64) NUPS_NORM((VEC <= 4 ? 16 : 32), (VEC <= 4 ? 4 : 2), 1)
        else if (chunks <= 128) NUPS_NORM(128, 1, 4)
        else if (chunks <= 256) NUPS_NORM(128, 2, 4)
        else if (chunks <= 512) NUPS_NORM(256, 2, 4)
        else if (chunks <= 1024) NUPS_NORM(512, 2, 2)
        else if (chunks <= 2048) NUPS_NORM(1024, 2, 1)
        else if (chunks <= 4096) NUPS_NORM(1024, 4, 1)
        else nups_launch_dependent(norm_long_kernel<X, VEC, KEYED>, grid_for(a.n, 1, (unsigned)s->sm_count * 2), 1024, 0, st, a, v);
    } else {
        // rows that 16-byte loads cannot read: pairs of 16-bit values where length and addresses are even, else single values.
        // Forward with one or two rows of a few chunks per lane: 600,000 rows of 17 floats 32 us (85 with a warp and four rows),
        // 400,000 rows of 34 bf16 24 us (63 by single values), 20,000 rows of 2046 bf16 41 us (55 by single values).
        if (chunks <= 16) NUPS_NORM(4, 4, 1)
        else if (chunks <= 32) NUPS_NORM(8, 4, 1)
        else if (chunks <= 64) NUPS_NORM(16, 4, 1)
        else if (chunks <= 128) NUPS_NORM(32, 4, 2)
        else if (chunks <= 256) NUPS_NORM(32, 8, (VEC == 1 && sizeof(X) == 2 ? 2 : 1))
        else if (chunks <= 512) NUPS_NORM(32, 16, 1)
        else if (chunks <= 1024) NUPS_NORM(128, 8, 2)
        else if (chunks <= 2048) NUPS_NORM(256, 8, 2)
        else if (chunks <= 4096) NUPS_NORM(256, 16, 1)
        else if (chunks <= 8192) NUPS_NORM(512, 16, 1)
        else if (chunks <= 16384) NUPS_NORM(1024, 16, 1)
        else nups_launch_dependent(norm_long_kernel<X, VEC, KEYED>, grid_for(a.n, 1, (unsigned)s->sm_count * 2), 1024, 0, st, a, v);
    }
#undef NUPS_NORM
    LAUNCH_CHECK(s);
    return NUPS_OK;
}

size_t stat_bytes(int x_type) { return x_type == NUPS_F64 ? 8 : 4; }

// weight and bias may be read VEC values at a time
int params_vec(const NormArgs& a, int x_type, int vec)
{
    const size_t run = (size_t)vec * (a.w_type == NUPS_F32 && x_type != NUPS_F64 ? 4 : type_bytes(x_type));
    const size_t need = run > 16 ? 16 : run;
    return suits(need, a.w, a.b);
}

bool w_type_fits(int x_type, int w_type) { return w_type == x_type || (w_type == NUPS_F32 && x_type != NUPS_F64); }
bool other_type_fits(int x_type, int t) { return t == x_type || (x_type == NUPS_F32 && (t == NUPS_F16 || t == NUPS_BF16)); }
bool eps_fits(int x_type, double eps) { return eps > 0 && eps < 1e30 && (x_type == NUPS_F64 || (float)eps > 0); }

// Do rows of `len` values of this type, `stride` apart, allow runs of `vec` values?
bool rows_allow(const void* p, int type, uint64_t stride, uint32_t len, int vec, uint64_t n)
{
    const size_t run = type_bytes(type) * vec, need = run > 16 ? 16 : run;
    return len % vec == 0 && suits(need, p) && (n <= 1 || stride % vec == 0);
}

}  // namespace

extern "C" nups_status nups_layer_norm(nups_store* s, const void* d_x, int x_type, uint64_t x_stride, uint64_t n, uint32_t len,
                                       const void* d_weight, const void* d_bias, int w_type, double eps, void* d_y, int y_type,
                                       uint64_t y_stride, void* d_mean, void* d_rstd, void* stream)
{
    if (!s || !type_known(x_type) || !other_type_fits(x_type, y_type) || !w_type_fits(x_type, w_type) || !eps_fits(x_type, eps)) return NUPS_EINVAL;
    if (len == 0 || len >= (1u << 28) || n >= (1ull << 32) || (n > 1 && (x_stride < len || y_stride < len))) return NUPS_EINVAL;
    if (x_stride >= (1ull << 32) || y_stride >= (1ull << 32)) return NUPS_EINVAL;
    if (n && (!d_x || !d_y)) return NUPS_EINVAL;
    if (!suits(type_bytes(x_type), d_x) || !suits(type_bytes(y_type), d_y) || !suits(type_bytes(w_type), d_weight, d_bias) ||
        !suits(stat_bytes(x_type), d_mean, d_rstd))
        return NUPS_EINVAL;
    nups_status rc = on_own_device(s);
    if (rc != NUPS_OK || n == 0) return rc;
    NormArgs a = {d_x, x_stride, d_y, y_stride, d_weight, d_bias, d_mean, d_rstd, n, len, y_type, w_type, 0, eps, nullptr, nullptr, s->st};
    const View v = {};
    cudaStream_t st = (cudaStream_t)stream;
    const int vec = (int)(16 / type_bytes(x_type));
    const bool wide = rows_allow(d_x, x_type, x_stride, len, vec, n) && rows_allow(d_y, y_type, y_stride, len, vec, n);
    const bool pairs = !wide && rows_allow(d_x, x_type, x_stride, len, 2, n) && rows_allow(d_y, y_type, y_stride, len, 2, n);    // 16-bit rows of even length
    a.w_vec = (wide && params_vec(a, x_type, vec)) || (pairs && params_vec(a, x_type, 2));
    switch (x_type) {
        case NUPS_F64: return wide ? launch_norm<double, 2, false>(s, a, v, st) : launch_norm<double, 1, false>(s, a, v, st);
        case NUPS_F32: return wide ? launch_norm<float, 4, false>(s, a, v, st) : launch_norm<float, 1, false>(s, a, v, st);
        case NUPS_F16: return wide ? launch_norm<__half, 8, false>(s, a, v, st) : pairs ? launch_norm<__half, 2, false>(s, a, v, st) : launch_norm<__half, 1, false>(s, a, v, st);
        default: return wide ? launch_norm<__nv_bfloat16, 8, false>(s, a, v, st) : pairs ? launch_norm<__nv_bfloat16, 2, false>(s, a, v, st) : launch_norm<__nv_bfloat16, 1, false>(s, a, v, st);
    }
}

extern "C" nups_status nups_pull_norm(nups_store* s, const uint32_t* d_keys, uint64_t n, const void* d_weight, const void* d_bias, double eps,
                                      void* d_y, int y_type, void* d_rows, void* d_mean, void* d_rstd, void* stream)
{
    if (!s) return NUPS_EINVAL;
    const int type = s->vb == 8 ? NUPS_F64 : NUPS_F32;
    if (!other_type_fits(type, y_type) || !eps_fits(type, eps) || n >= (1ull << 32) || (n && (!d_keys || !d_y))) return NUPS_EINVAL;
    if (!suits(16, d_y, d_rows) || !suits(4, d_keys) || !suits(type_bytes(type), d_weight, d_bias, d_mean, d_rstd)) return NUPS_EINVAL;
    nups_status rc = on_own_device(s);
    if (rc != NUPS_OK || n == 0) return rc;
    if (s->value_len >= (1u << 28)) return NUPS_EINVAL;     // positions within a row are 32 bits, and run some thousand past its end
    NormArgs a = {s->val, s->value_len, d_y, s->value_len, d_weight, d_bias, d_mean, d_rstd, n, s->value_len, y_type, type, 0, eps, d_keys, d_rows, s->st};
    a.w_vec = params_vec(a, type, type == NUPS_F64 ? 2 : 4);
    const View v = nups_view(s);
    const cudaStream_t st = (cudaStream_t)stream;
    nups_time_begin(s, st, NUPS_TIMED_PULL);
    rc = type == NUPS_F64 ? launch_norm<double, 2, true>(s, a, v, st) : launch_norm<float, 4, true>(s, a, v, st);
    nups_time_end(s, st);
    return rc;
}

// ---------------------------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------------------------
namespace {

struct GradArgs {
    const void* x;
    uint64_t xs;
    const void* dy;
    uint64_t dys;
    const void *mean, *rstd, *w;
    void* dx;
    uint64_t dxs;
    void* part;                // [blocks][2][len] sums of dy h and of dy over a block's rows; NULL: not wanted
    uint64_t n;
    uint32_t len;
    int dy_type, w_type, w_vec;
    DevStat* st;
};

// Rows that are added one after the other before the sums go to (and are added in) the block's part of scratch: the rounding of a
// sum over n rows grows with this number and with n / (blocks * SUM_RUN), not with n / blocks (3M rows of 300 equal values: 1.5e-6 of the
// sum, 4.9e-5 with one run per block).  With 64 rows 60,000 rows of 1000 bf16 took 89 us, with 128 they take 79.
constexpr uint32_t SUM_RUN = 128;
// N sums into a block's part of scratch: stored the first time, added after that.  N loads in flight, not all of a thread's, so that
// this takes no registers from the loop.
template <int N, class A> __device__ __forceinline__ void put_sums(A* to, A* sums, bool before)
{
#pragma unroll
    for (int j = 0; j < N; ++j) {
        to[j] = before ? to[j] + sums[j] : sums[j];
        sums[j] = 0;
    }
    asm volatile("" ::: "memory");
}

// One pass: a team holds x and dy of ROWS rows in registers and, over SUM_RUN of its rows, its columns' shares of dweight and dbias
// (SHARED: in shared memory, where 64 registers a thread leave no room; each thread has its own columns there).
// Short rows of floats by 16 bytes: three blocks per multiprocessor, as many as grad_blocks gives (the compiler would take 96
// registers, for two).  The others as the compiler sees fit.
constexpr int grad_min_blocks(int tpr, int vec, int ept, size_t d) { return tpr <= 32 && vec == 4 && (ept == 4 || d == 2) ? 3 : 0; }
template <class X, class D, int VEC, int TPR, int CH, int ROWS>
__global__ void __launch_bounds__(team_block(TPR), grad_min_blocks(TPR, VEC, CH * VEC, sizeof(D))) norm_grad_kernel(GradArgs a)
{
    typedef typename Acc<X>::type A;
    constexpr int BLOCK = team_block(TPR), TEAMS = BLOCK / TPR, WARPS = BLOCK / 32, EPT = CH * VEC;
    constexpr bool SHARED = TPR == 1024;
    extern __shared__ char dynamic[];                       // SHARED: [2][len] sums
    __shared__ A shared[TPR > 32 ? 4 * ROWS * WARPS : WARPS * TPR * EPT];
    grid_dependency_wait();
    const int t = threadIdx.x % TPR, team = threadIdx.x / TPR;
    A w[CH][VEC], dw[CH][VEC], db[CH][VEC];
    A* const sum_w = (A*)dynamic;
    A* const sum_b = sum_w + (SHARED ? CH * VEC * TPR : 0);
    if (!SHARED) load_params<X, A, VEC, TPR, CH>(a.w, a.w_type, a.w_vec, a.len, t, (A)1, w);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            if (SHARED) sum_w[value_at<TPR, VEC>(c, t) + j] = sum_b[value_at<TPR, VEC>(c, t) + j] = 0;
            else dw[c][j] = db[c][j] = 0;
        }
    const A inv_len = (A)1 / (A)a.len;
    A* const out = (A*)a.part + (uint64_t)blockIdx.x * 2 * a.len;
    bool before = false;
    auto put_down = [&] {                                   // the whole block
        if (TPR > 32) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const uint32_t at = value_at<TPR, VEC>(c, t);
                if (at < a.len) {
                    put_sums<VEC>(out + at, SHARED ? sum_w + at : dw[c], before);
                    put_sums<VEC>(out + a.len + at, SHARED ? sum_b + at : db[c], before);
                }
            }
        } else {
            // teams of a warp by shuffles, warps through shared memory; first dweight, then dbias
            A* mine = shared + (threadIdx.x >> 5) * TPR * EPT;
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                __syncthreads();
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        A p = which ? db[c][j] : dw[c][j];
#pragma unroll
                        for (int o = TPR; o < 32; o <<= 1) p += __shfl_xor_sync(0xFFFFFFFFu, p, o);
                        if ((threadIdx.x & 31) < TPR) mine[value_at<TPR, VEC>(c, t) + j] = p;
                        if (which) db[c][j] = 0;
                        else dw[c][j] = 0;
                    }
                __syncthreads();
                for (uint32_t i = threadIdx.x; i < a.len; i += BLOCK) {
                    A sum = 0;
#pragma unroll
                    for (int k = 0; k < WARPS; ++k) sum += shared[k * TPR * EPT + i];
                    out[which * a.len + i] = before ? out[which * a.len + i] + sum : sum;
                }
            }
        }
        before = true;
    };
    int turn = 0;
    uint64_t base = (uint64_t)blockIdx.x * (TEAMS * ROWS);
    do {
        for (int end = turn + SUM_RUN / ROWS; turn < end && base < a.n; base += (uint64_t)gridDim.x * (TEAMS * ROWS), ++turn) {
            Pack<X, VEC> x[ROWS][CH];
            Pack<D, VEC> dy[ROWS][CH];
            A mean[ROWS], rstd[ROWS], s1[ROWS], s2[ROWS];
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                const uint64_t row = base + k * TEAMS + team;
                const bool in = row < a.n;
                mean[k] = in ? ((const A*)a.mean)[row] : (A)0;
                rstd[k] = in ? ((const A*)a.rstd)[row] : (A)0;
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const uint32_t at = value_at<TPR, VEC>(c, t);
                    if (in && at < a.len) {
                        x[k][c] = load_pack<X, VEC>((const X*)a.x + row * a.xs + at);
                        dy[k][c] = load_pack<D, VEC>((const D*)a.dy + row * a.dys + at);
                    } else {
                        x[k][c] = Pack<X, VEC>{};
                        dy[k][c] = Pack<D, VEC>{};
                    }
                }
            }
            A a1[ROWS][2], a2[ROWS][2];
#pragma unroll
            for (int k = 0; k < ROWS; ++k) a1[k][0] = a1[k][1] = a2[k][0] = a2[k][1] = 0;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const uint32_t at = value_at<TPR, VEC>(c, t);
                if (at < a.len) {
                    A wc[1][VEC], dwc[VEC], dbc[VEC];
                    if (SHARED) {
                        load_params_at<X, A, VEC>(a.w, a.w_type, a.w_vec, at, (A)1, wc);
#pragma unroll
                        for (int j = 0; j < VEC; ++j) { dwc[j] = sum_w[at + j]; dbc[j] = sum_b[at + j]; }
                    }
                    // rows that are not there have dy = 0 and rstd = 0: they add nothing
#pragma unroll
                    for (int k = 0; k < ROWS; ++k) {
                        const A minus = -mean[k];
                        A h[VEC], d[VEC];
                        unpack<A>(x[k][c], h);
                        unpack<A>(dy[k][c], d);
                        run_add<VEC, true>(h, h, &minus);
                        run_scale<VEC>(h, h, rstd[k]);
                        run_fma<VEC, false, false, false>(SHARED ? dwc : dw[c], d, h, SHARED ? dwc : dw[c]);
                        run_add<VEC, false>(SHARED ? dbc : db[c], SHARED ? dbc : db[c], d);
                        run_mul<VEC>(d, d, SHARED ? wc[0] : w[c]);
                        sum_run<VEC>(a1[k], d);
                        sum_run_of_products<VEC>(a2[k], d, h);
                    }
                    if (SHARED)
#pragma unroll
                        for (int j = 0; j < VEC; ++j) { sum_w[at + j] = dwc[j]; sum_b[at + j] = dbc[j]; }
                }
            }
#pragma unroll
            for (int k = 0; k < ROWS; ++k) { s1[k] = a1[k][0] + a1[k][1]; s2[k] = a2[k][0] + a2[k][1]; }
            if (!a.dx) continue;                                // the same for the whole grid
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                s1[k] = team_sum<(TPR < 32 ? TPR : 32)>(s1[k]);
                s2[k] = team_sum<(TPR < 32 ? TPR : 32)>(s2[k]);
            }
            if (TPR > 32) {
                A* st = shared + (turn & 1) * 2 * ROWS * WARPS;
                const int lane = t & 31;
                if (lane == 0)
#pragma unroll
                    for (int k = 0; k < ROWS; ++k) { st[k * WARPS + (t >> 5)] = s1[k]; st[(ROWS + k) * WARPS + (t >> 5)] = s2[k]; }
                __syncthreads();
                // lanes [i WARPS, (i + 1) WARPS) take sum i of the 2 ROWS, 32 / WARPS sums at a time
                constexpr int AT_ONCE = 32 / WARPS < 2 * ROWS ? 32 / WARPS : 2 * ROWS;
#pragma unroll
                for (int i0 = 0; i0 < 2 * ROWS; i0 += AT_ONCE) {
                    const A sum = team_sum<WARPS>(st[(i0 + (lane / WARPS) % AT_ONCE) * WARPS + lane % WARPS]);
#pragma unroll
                    for (int i = 0; i < AT_ONCE; ++i) {
                        const A r = __shfl_sync(0xFFFFFFFFu, sum, i * WARPS);
                        if (i0 + i < ROWS) s1[i0 + i] = r;
                        else s2[i0 + i - ROWS] = r;
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const uint32_t at = value_at<TPR, VEC>(c, t);
                if (at < a.len) {
                    A wc[1][VEC];
                    if (SHARED) load_params_at<X, A, VEC>(a.w, a.w_type, a.w_vec, at, (A)1, wc);
#pragma unroll
                    for (int k = 0; k < ROWS; ++k) {
                        const uint64_t row = base + k * TEAMS + team;
                        // rstd (g - mean(g) - h mean(g h)), the two means with the factor rstd already
                        const A minus = -mean[k], m1 = -s1[k] * inv_len * rstd[k], m2 = -s2[k] * inv_len * rstd[k];
                        A h[VEC], d[VEC];
                        unpack<A>(x[k][c], h);
                        unpack<A>(dy[k][c], d);
                        run_add<VEC, true>(h, h, &minus);
                        run_scale<VEC>(h, h, rstd[k]);
                        run_mul<VEC>(d, d, SHARED ? wc[0] : w[c]);
                        run_fma<VEC, false, true, true>(h, h, &m2, &m1);
                        run_fma<VEC, false, true, false>(d, d, &rstd[k], h);
                        if (row < a.n) store_values<X, VEC>((X*)a.dx + row * a.dxs + at, d);
                    }
                }
            }
        }
        if (a.part) put_down();
    } while (base < a.n);
}

// Rows above 1 KB: x and dy come through a ring in shared memory, as in norm_ring_kernel, and are read there twice.
// (16,384 rows of 4096 bf16: 90 us with the rows in registers.)  As many blocks per multiprocessor as grad_blocks gives: with the compiler's
// own choice of registers the same rows take 87 us instead of 84, 60,000 of 1000 bf16 81 instead of 79.
template <class X, class D, int TPR, int CH, int ROWS, int STAGES>
__global__ void __launch_bounds__(TPR, 512 / TPR) norm_grad_ring_kernel(GradArgs a)
{
    typedef typename Acc<X>::type A;
    constexpr int VEC = 16 / sizeof(X), WARPS = TPR / 32;
    extern __shared__ __align__(128) char ring[];
    __shared__ A shared[4 * ROWS * WARPS];
    __shared__ uint64_t bars[STAGES];
    const int t = threadIdx.x;
    const uint32_t x_bytes = a.len * sizeof(X), d_bytes = a.len * sizeof(D), stage_bytes = (x_bytes + d_bytes) * ROWS;
    const uint64_t step = (uint64_t)gridDim.x * ROWS, first = (uint64_t)blockIdx.x * ROWS;
    auto bar = [&](uint32_t s) { return smem_address(&bars[s]); };
    if (t == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(bar(s), 1);
        mbar_init_visible();
    }
    grid_dependency_wait();
    auto issue = [&](uint32_t i) {                          // the block's group i; one thread
        const uint64_t base = first + i * step;
        if (base >= a.n) return;
        const uint32_t rows = (uint32_t)min((uint64_t)ROWS, a.n - base), s = i % STAGES, to = smem_address(ring) + s * stage_bytes, to_d = to + ROWS * x_bytes;
        mbar_expect(bar(s), rows * (x_bytes + d_bytes));
        if (a.xs == a.len) bulk_load(to, (const X*)a.x + base * a.xs, rows * x_bytes, bar(s));
        else
            for (uint32_t k = 0; k < rows; ++k) bulk_load(to + k * x_bytes, (const X*)a.x + (base + k) * a.xs, x_bytes, bar(s));
        if (a.dys == a.len) bulk_load(to_d, (const D*)a.dy + base * a.dys, rows * d_bytes, bar(s));
        else
            for (uint32_t k = 0; k < rows; ++k) bulk_load(to_d + k * d_bytes, (const D*)a.dy + (base + k) * a.dys, d_bytes, bar(s));
    };
    if (t == 0)
        for (uint32_t i = 0; i + 1 < STAGES; ++i) issue(i);
    A w[CH][VEC], dw[CH][VEC], db[CH][VEC];
    load_params<X, A, VEC, TPR, CH>(a.w, a.w_type, a.w_vec, a.len, t, (A)1, w);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < VEC; ++j) dw[c][j] = db[c][j] = 0;
    const A inv_len = (A)1 / (A)a.len;
    A* const out = (A*)a.part + (uint64_t)blockIdx.x * 2 * a.len;
    bool before = false;
    auto put_down = [&] {                                   // as in norm_grad_kernel
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const uint32_t at = value_at<TPR, VEC>(c, t);
            if (at < a.len) {
                put_sums<VEC>(out + at, dw[c], before);
                put_sums<VEC>(out + a.len + at, db[c], before);
            }
        }
        before = true;
    };
    __syncthreads();                                        // the barriers are there
    uint32_t i = 0;
    bool ok = true;
    uint64_t base = first;
    do {
        for (uint32_t end = i + SUM_RUN / ROWS; i < end && base < a.n; base += step, ++i) {
            const uint32_t s = i % STAGES;
            const X* x = (const X*)(ring + s * stage_bytes);
            const D* dy = (const D*)(ring + s * stage_bytes + ROWS * x_bytes);
            A mean[ROWS], rstd[ROWS], s1[ROWS], s2[ROWS];
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                mean[k] = base + k < a.n ? ((const A*)a.mean)[base + k] : (A)0;
                rstd[k] = base + k < a.n ? ((const A*)a.rstd)[base + k] : (A)0;
            }
            ok = mbar_wait(bar(s), (i / STAGES) & 1);
            auto hat = [&](int k, uint32_t at, A* h, A* d) {
                const A minus = -mean[k];
                unpack<A>(load_pack<X, VEC>(x + k * a.len + at), h);
                unpack<A>(load_pack<D, VEC>(dy + k * a.len + at), d);
                run_add<VEC, true>(h, h, &minus);
                run_scale<VEC>(h, h, rstd[k]);
            };
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                A a1[2] = {0, 0}, a2[2] = {0, 0};
                if (base + k < a.n)                             // the same for the whole block
#pragma unroll
                    for (int c = 0; c < CH; ++c) {
                        const uint32_t at = value_at<TPR, VEC>(c, t);
                        if (at < a.len) {
                            A h[VEC], d[VEC];
                            hat(k, at, h, d);
                            run_fma<VEC, false, false, false>(dw[c], d, h, dw[c]);
                            run_add<VEC, false>(db[c], db[c], d);
                            run_mul<VEC>(d, d, w[c]);
                            sum_run<VEC>(a1, d);
                            sum_run_of_products<VEC>(a2, d, h);
                        }
                    }
                s1[k] = a1[0] + a1[1];
                s2[k] = a2[0] + a2[1];
            }
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                s1[k] = team_sum<32>(s1[k]);
                s2[k] = team_sum<32>(s2[k]);
            }
            A* st = shared + (i & 1) * 2 * ROWS * WARPS;
            const int lane = t & 31;
            if (lane == 0)
#pragma unroll
                for (int k = 0; k < ROWS; ++k) { st[k * WARPS + (t >> 5)] = s1[k]; st[(ROWS + k) * WARPS + (t >> 5)] = s2[k]; }
            if (__syncthreads_or(!ok)) { ok = false; break; }
            if (t == 0) issue(i + STAGES - 1);                  // every thread is done with the group before this one
            if (!a.dx) continue;
            constexpr int AT_ONCE = 32 / WARPS < 2 * ROWS ? 32 / WARPS : 2 * ROWS;
#pragma unroll
            for (int i0 = 0; i0 < 2 * ROWS; i0 += AT_ONCE) {
                const A sum = team_sum<WARPS>(st[(i0 + (lane / WARPS) % AT_ONCE) * WARPS + lane % WARPS]);
#pragma unroll
                for (int q = 0; q < AT_ONCE; ++q) {
                    const A r = __shfl_sync(0xFFFFFFFFu, sum, q * WARPS);
                    if (i0 + q < ROWS) s1[i0 + q] = r;
                    else s2[i0 + q - ROWS] = r;
                }
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const uint32_t at = value_at<TPR, VEC>(c, t);
                if (at < a.len)
#pragma unroll
                    for (int k = 0; k < ROWS; ++k) {
                        const A m1 = -s1[k] * inv_len * rstd[k], m2 = -s2[k] * inv_len * rstd[k];
                        A h[VEC], d[VEC];
                        hat(k, at, h, d);
                        run_mul<VEC>(d, d, w[c]);
                        run_fma<VEC, false, true, true>(h, h, &m2, &m1);
                        run_fma<VEC, false, true, false>(d, d, &rstd[k], h);
                        if (base + k < a.n) store_values<X, VEC>((X*)a.dx + (base + k) * a.dxs + at, d);
                    }
            }
        }
        if (a.part) put_down();
    } while (ok && base < a.n);
    if (!ok) {                                              // a copy did not come: say so, and leave none in flight
        atomicCAS(&a.st->status, 0, NUPS_ETIMEOUT);
        if (t == 0)
            for (uint32_t k = i + 1; k < i + STAGES - 1; ++k)
                if (first + k * step < a.n) mbar_wait(bar(k % STAGES), (k / STAGES) & 1);
    }
}

// Rows too long for registers, first pass: a block per row leaves mean(g) and mean(g h).
template <class X, int VEC>
__global__ void __launch_bounds__(1024) norm_grad_sums_kernel(GradArgs a, typename Acc<X>::type* sums)
{
    typedef typename Acc<X>::type A;
    __shared__ double shared[32];
    grid_dependency_wait();
    for (uint64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const A mean = ((const A*)a.mean)[row], rstd = ((const A*)a.rstd)[row];
        double s1 = 0, s2 = 0;                              // as in norm_long_kernel
        for (uint32_t at = threadIdx.x * VEC; at < a.len; at += 1024 * VEC) {
            A x[VEC], g[VEC], w[1][VEC], run1 = 0, run2 = 0;
            unpack<A>(load_pack<X, VEC>((const X*)a.x + row * a.xs + at), x);
            load_chunk<X, A, VEC>(a.dy, a.dy_type, row * a.dys + at, g);
            load_params_at<X, A, VEC>(a.w, a.w_type, a.w_vec, at, (A)1, w);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const A gj = g[j] * w[0][j];
                run1 += gj;
                run2 += gj * ((x[j] - mean) * rstd);
            }
            s1 += (double)run1;
            s2 += (double)run2;
        }
        s1 = block_sum(s1, shared);
        s2 = block_sum(s2, shared);
        if (threadIdx.x == 0) { sums[2 * row] = (A)(s1 / a.len); sums[2 * row + 1] = (A)(s2 / a.len); }
    }
}
// Second pass: a warp per run of 32 * VEC columns of a stretch of rows (blockIdx.y of gridDim.y).
template <class X, int VEC>
__global__ void __launch_bounds__(256) norm_grad_apply_kernel(GradArgs a, const typename Acc<X>::type* sums)
{
    typedef typename Acc<X>::type A;
    grid_dependency_wait();
    const uint32_t at = (blockIdx.x * 256 + threadIdx.x) * VEC;
    if (at >= a.len) return;
    A w[1][VEC], dw[VEC], db[VEC];
    load_params_at<X, A, VEC>(a.w, a.w_type, a.w_vec, at, (A)1, w);
#pragma unroll
    for (int j = 0; j < VEC; ++j) dw[j] = db[j] = 0;
    A* const out = (A*)a.part + (uint64_t)blockIdx.y * 2 * a.len + at;
    bool before = false;
    auto put_down = [&] {                                   // as in norm_grad_kernel
        put_sums<VEC>(out, dw, before);
        put_sums<VEC>(out + a.len, db, before);
        before = true;
    };
    uint32_t run = 0;
    for (uint64_t row = blockIdx.y; row < a.n; row += gridDim.y, ++run) {
        if (a.part && run == SUM_RUN) { put_down(); run = 0; }
        const A mean = ((const A*)a.mean)[row], rstd = ((const A*)a.rstd)[row];
        A x[VEC], g[VEC], d[VEC];
        unpack<A>(load_pack<X, VEC>((const X*)a.x + row * a.xs + at), x);
        load_chunk<X, A, VEC>(a.dy, a.dy_type, row * a.dys + at, g);
        const A s1 = a.dx ? sums[2 * row] : (A)0, s2 = a.dx ? sums[2 * row + 1] : (A)0;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const A h = (x[j] - mean) * rstd;
            dw[j] += g[j] * h;
            db[j] += g[j];
            d[j] = (g[j] * w[0][j] - s1 - h * s2) * rstd;
        }
        if (a.dx) store_values<X, VEC>((X*)a.dx + row * a.dxs + at, d);
    }
    if (a.part) put_down();
}

// dweight and dbias: the blocks' sums, added in a fixed order.  32 columns and 32 runs of blocks per block of threads.
template <class A, class T>
__global__ void __launch_bounds__(1024) norm_grad_join_kernel(const A* part, uint32_t blocks, uint32_t len, T* dw, T* db)
{
    __shared__ A shared[32][33];
    grid_dependency_wait();
    const uint32_t col = blockIdx.x * 32 + (threadIdx.x & 31), run = threadIdx.x >> 5;
    T* out = blockIdx.y ? db : dw;
    if (!out) return;
    A sum = 0;
    if (col < len)
#pragma unroll 8
        for (uint32_t k = run; k < blocks; k += 32) sum += __ldcg(part + ((uint64_t)k * 2 + blockIdx.y) * len + col);
    shared[run][threadIdx.x & 31] = sum;
    __syncthreads();
    if (run == 0 && col < len) {
        sum = 0;
#pragma unroll
        for (int k = 0; k < 32; ++k) sum += shared[k][threadIdx.x];
        out[col] = narrow<T>(sum);
    }
}

// The longest rows that a team holds; longer ones take two passes over x and dy.
uint32_t grad_long_from(int type) { return type == NUPS_F64 ? 4096 : 16384; }

// Blocks that leave sums: a rule on the sizes alone, so that the order of the additions is theirs too.
unsigned grad_blocks(const nups_store* s, uint64_t n, uint32_t len, int type)
{
    const unsigned sm = (unsigned)s->sm_count;
    const uint32_t bytes = len * (uint32_t)type_bytes(type);
    if (len > grad_long_from(type)) return grid_for(n, 16, 32);
    return grid_for(n, bytes <= 128 ? 64 : bytes <= 1024 ? 8 : 2, sm * (bytes <= 1024 ? 3 : bytes <= 4096 ? 4 : bytes <= (type_bytes(type) == 2 ? 8192u : 16384u) ? 2 : 1));
}
uint64_t grad_part_bytes(const nups_store* s, uint64_t n, uint32_t len, int type)
{
    return (uint64_t)grad_blocks(s, n, len, type) * 2 * len * (type == NUPS_F64 ? 8 : 4);
}

template <class X, class D, int VEC>
nups_status launch_grad(nups_store* s, GradArgs a, int x_type, void* d_dw, void* d_db, char* scratch, cudaStream_t st)
{
    typedef typename Acc<X>::type A;
    const uint32_t len = a.len;
    const unsigned blocks = grad_blocks(s, a.n, len, x_type);
    const uint32_t chunks = (len + VEC - 1) / VEC;
#define NUPS_GRAD(TPR_, CH_, ROWS_)                                                                                       \
    {                                                                                                                     \
        const unsigned smem = TPR_ == 1024 ? 2 * TPR_ * CH_ * VEC * (unsigned)sizeof(A) : 0;                              \
        if (smem > 48 * 1024) CK(cudaFuncSetAttribute(norm_grad_kernel<X, D, VEC, TPR_, CH_, ROWS_>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem)); \
        nups_launch_dependent(norm_grad_kernel<X, D, VEC, TPR_, CH_, ROWS_>, blocks, team_block(TPR_), smem, st, a);      \
    }
#define NUPS_GRAD_RING(TPR_, CH_, ROWS_, STAGES_)                                                                                           \
    {                                                                                                                                      \
        constexpr size_t largest = (size_t)STAGES_ * ROWS_ * TPR_ * CH_ * VEC * (sizeof(X) + sizeof(D));                                   \
        const size_t smem = (size_t)STAGES_ * ROWS_ * len * (sizeof(X) + sizeof(D));                                                       \
        static RingLimits known;                                                                                                           \
        if (!ring_blocks(known, s->device, norm_grad_ring_kernel<X, D, TPR_, CH_, ROWS_, STAGES_>, TPR_, largest, smem))                   \
            return nups_cuda_fail(cudaGetLastError(), "norm_grad_ring_kernel");                                                            \
        nups_launch_dependent(norm_grad_ring_kernel<X, D, TPR_, CH_, ROWS_, STAGES_>, blocks, TPR_, smem, st, a);                          \
    }
    bool through_ring = false;
    if constexpr (VEC * sizeof(X) == 16) {
        // fewer rows: every block has one group, nothing to run ahead of
        through_ring = chunks > 64 && chunks <= (sizeof(X) == 2 ? 1024 : 2048) && a.n > (uint64_t)s->sm_count && len * sizeof(D) % 16 == 0 && ((uintptr_t)a.dy & 15) == 0 &&
                       a.dys * sizeof(D) % 16 == 0;
        if (through_ring) {
            if (chunks <= 128) NUPS_GRAD_RING(128, 1, 4, 3)
            else if (chunks <= 256) NUPS_GRAD_RING(128, 2, 2, 3)
            else if (chunks <= 512) NUPS_GRAD_RING(256, 2, 2, 3)
            else if constexpr (sizeof(X) == 2) NUPS_GRAD_RING(512, 2, 2, 3)
            else if (chunks <= 1024) NUPS_GRAD_RING(256, 4, 1, 3)
            else NUPS_GRAD_RING(512, 4, 1, 3)
        }
    }
#undef NUPS_GRAD_RING
    if (through_ring) {
        // launched above
    } else if (len > grad_long_from(x_type)) {
        A* sums = (A*)(scratch + (a.part ? (grad_part_bytes(s, a.n, len, x_type) + 255) / 256 * 256 : 0));
        if (a.dx) {
            nups_launch_dependent(norm_grad_sums_kernel<X, VEC>, grid_for(a.n, 1, (unsigned)s->sm_count * 2), 1024, 0, st, a, sums);
            LAUNCH_CHECK(s);
        }
        nups_launch_dependent(norm_grad_apply_kernel<X, VEC>, dim3(grid_for(len, 256 * VEC), blocks), 256, 0, st, a, (const A*)sums);
    }
    else if constexpr (VEC * sizeof(X) == 16) {
        if (chunks <= 4) NUPS_GRAD(4, 1, 4)
        else if (chunks <= 8) NUPS_GRAD(8, 1, 4)
        else if (chunks <= 16) NUPS_GRAD(16, 1, 4)
        else if (chunks <= 32) NUPS_GRAD(32, 1, 4)
        else if (chunks <= 64) NUPS_GRAD(32, 2, 2)
        else if (chunks <= 128) NUPS_GRAD(128, 1, 4)
        else if (chunks <= 256) NUPS_GRAD(128, 2, 2)
        else if (chunks <= 512) NUPS_GRAD(256, 2, 2)
        else if (chunks <= 1024) NUPS_GRAD(512, 2, 1)
        else if (chunks <= 2048) NUPS_GRAD(1024, 2, 1)
        else if constexpr (VEC == 4) NUPS_GRAD(1024, 4, 1)
    } else {
        // as forward: 600,000 rows of 17 floats 40 us (92 with a warp and four rows), 400,000 rows of 34 bf16 34 us (83 by single values)
        if (chunks <= 16) NUPS_GRAD(4, 4, 2)
        else if (chunks <= 32) NUPS_GRAD(8, 4, 2)
        else if (chunks <= 64) NUPS_GRAD(16, 4, 2)
        else if (chunks <= 128) NUPS_GRAD(32, 4, 2)
        else if (chunks <= 256) NUPS_GRAD(32, 8, 1)
        else if (chunks <= 512) NUPS_GRAD(32, 16, 1)
        else if (chunks <= 1024) NUPS_GRAD(128, 8, 1)
        else if (chunks <= 2048) NUPS_GRAD((VEC == 1 ? 128 : 256), (VEC == 1 ? 16 : 8), 1)
        else if (chunks <= 4096) NUPS_GRAD((VEC == 1 ? 256 : 512), (VEC == 1 ? 16 : 8), 1)
        else if constexpr (sizeof(A) == 4 && VEC == 1) {
            if (chunks <= 8192) NUPS_GRAD(512, 16, 1)
            else NUPS_GRAD(1024, 16, 1)
        } else if constexpr (VEC == 2) NUPS_GRAD(1024, 8, 1)
    }
#undef NUPS_GRAD
    LAUNCH_CHECK(s);
    if (a.part) {
        const dim3 grid((len + 31) / 32, 2);
        bool wide_params = false;                           // fp32 parameters of 16-bit rows
        if constexpr (sizeof(X) == 2) {
            wide_params = a.w_type == NUPS_F32;
            if (wide_params) nups_launch_dependent(norm_grad_join_kernel<A, float>, grid, 1024, 0, st, (const A*)a.part, blocks, len, (float*)d_dw, (float*)d_db);
        }
        if (!wide_params) nups_launch_dependent(norm_grad_join_kernel<A, X>, grid, 1024, 0, st, (const A*)a.part, blocks, len, (X*)d_dw, (X*)d_db);
        LAUNCH_CHECK(s);
    }
    return NUPS_OK;
}

}  // namespace

extern "C" nups_status nups_layer_norm_grad_scratch(nups_store* s, uint64_t n, uint32_t len, int x_type, uint64_t* h_bytes_out)
{
    if (!s || !h_bytes_out || !type_known(x_type) || len == 0 || len >= (1u << 28) || n >= (1ull << 32)) return NUPS_EINVAL;
    uint64_t bytes = (grad_part_bytes(s, n, len, x_type) + 255) / 256 * 256;
    if (len > grad_long_from(x_type)) bytes += 2 * n * (x_type == NUPS_F64 ? 8 : 4);
    *h_bytes_out = bytes;
    return NUPS_OK;
}

extern "C" nups_status nups_layer_norm_grad(nups_store* s, const void* d_x, int x_type, uint64_t x_stride, const void* d_dy, int dy_type,
                                            uint64_t dy_stride, uint64_t n, uint32_t len, const void* d_mean, const void* d_rstd,
                                            const void* d_weight, int w_type, void* d_dx, uint64_t dx_stride, void* d_dweight,
                                            void* d_dbias, void* d_scratch, uint64_t scratch_bytes, void* stream)
{
    if (!s || !type_known(x_type) || !other_type_fits(x_type, dy_type) || !w_type_fits(x_type, w_type)) return NUPS_EINVAL;
    if (len == 0 || len >= (1u << 28) || n >= (1ull << 32) || (n > 1 && (x_stride < len || dy_stride < len || (d_dx && dx_stride < len)))) return NUPS_EINVAL;
    if (x_stride >= (1ull << 32) || dy_stride >= (1ull << 32) || dx_stride >= (1ull << 32)) return NUPS_EINVAL;
    if (n && (!d_x || !d_dy || !d_mean || !d_rstd)) return NUPS_EINVAL;
    if (!suits(type_bytes(x_type), d_x, d_dx) || !suits(type_bytes(dy_type), d_dy) || !suits(type_bytes(w_type), d_weight, d_dweight, d_dbias) ||
        !suits(stat_bytes(x_type), d_mean, d_rstd))
        return NUPS_EINVAL;
    const bool sums = d_dweight || d_dbias;
    const bool needs = n && (sums || (d_dx && len > grad_long_from(x_type)));
    uint64_t bytes = 0;
    nups_layer_norm_grad_scratch(s, n, len, x_type, &bytes);
    if (needs && (!d_scratch || scratch_bytes < bytes || !suits(256, d_scratch))) return NUPS_EINVAL;
    nups_status rc = on_own_device(s);
    if (rc != NUPS_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    if (n == 0) {
        if (d_dweight) CK(cudaMemsetAsync(d_dweight, 0, (size_t)len * type_bytes(w_type), st));
        if (d_dbias) CK(cudaMemsetAsync(d_dbias, 0, (size_t)len * type_bytes(w_type), st));
        return NUPS_OK;
    }
    if (!sums && !d_dx) return NUPS_OK;
    GradArgs a = {d_x, x_stride, d_dy, dy_stride, d_mean, d_rstd, d_weight, d_dx, dx_stride, sums ? d_scratch : nullptr, n, len, dy_type, w_type, 0, s->st};
    const int vec = (int)(16 / type_bytes(x_type));
    const bool wide = rows_allow(d_x, x_type, x_stride, len, vec, n) && rows_allow(d_dy, dy_type, dy_stride, len, vec, n) &&
                      (!d_dx || rows_allow(d_dx, x_type, dx_stride, len, vec, n));
    const bool pairs = !wide && rows_allow(d_x, x_type, x_stride, len, 2, n) && rows_allow(d_dy, dy_type, dy_stride, len, 2, n) &&
                       (!d_dx || rows_allow(d_dx, x_type, dx_stride, len, 2, n));           // 16-bit rows of even length
    const size_t run = (size_t)(pairs ? 2 : vec) * (w_type == NUPS_F32 && x_type != NUPS_F64 ? 4 : type_bytes(x_type));
    a.w_vec = (wide || pairs) && suits(run > 16 ? 16 : run, d_weight);
    char* scratch = (char*)d_scratch;
#define NUPS_LAUNCH(X_, D_, V_) (wide ? launch_grad<X_, D_, V_>(s, a, x_type, d_dweight, d_dbias, scratch, st) : launch_grad<X_, D_, 1>(s, a, x_type, d_dweight, d_dbias, scratch, st))
#define NUPS_LAUNCH16(X_) (!wide && pairs ? launch_grad<X_, X_, 2>(s, a, x_type, d_dweight, d_dbias, scratch, st) : NUPS_LAUNCH(X_, X_, 8))
    switch (x_type) {
        case NUPS_F64: return NUPS_LAUNCH(double, double, 2);
        case NUPS_F32: return dy_type == NUPS_F32 ? NUPS_LAUNCH(float, float, 4) : dy_type == NUPS_F16 ? NUPS_LAUNCH(float, __half, 4) : NUPS_LAUNCH(float, __nv_bfloat16, 4);
        case NUPS_F16: return NUPS_LAUNCH16(__half);
        default: return NUPS_LAUNCH16(__nv_bfloat16);
    }
#undef NUPS_LAUNCH16
#undef NUPS_LAUNCH
}
