// Layer norm of dense rows and of pulled rows, and its backward pass.
//
// y = (x - mean) rstd w + b is bound by memory: x is read once, y written once, some eight operations a value.  A row is held in
// the registers of a team of TPR threads (EPT values each), so the variance is taken about the mean in a second pass over
// registers, not as a difference of sums; w and b stay in registers while a team walks its rows.  Teams of up to 32 threads
// reduce by shuffles; a block that is one team merges its warps' (sum, sum of squares about the warp's own mean) with one
// barrier per row (Chan's formula for the variance of a union).
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
// Mean and reciprocal deviation of the row that the team holds in x (zero beyond len).
template <class A, int VEC, int TPR, int CH>
__device__ __forceinline__ void row_stats(const A (&x)[CH][VEC], uint32_t len, A eps, int t, int turn, A* shared, A& mean, A& rstd)
{
    constexpr int WARPS = TPR / 32;
    A sum = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < VEC; ++j) sum += x[c][j];
    sum = team_sum<(TPR < 32 ? TPR : 32)>(sum);
    A about;                                               // the mean that the squares are taken about: the team's, or the warp's
    uint32_t held = len;
    if (TPR > 32) {
        held = 0;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const uint32_t at = value_at<TPR, VEC>(c, t & ~31);
            held += at < len ? min((uint32_t)(32 * VEC), len - at) : 0u;
        }
        about = held ? sum / (A)held : (A)0;
    } else {
        about = sum / (A)len;
    }
    A sq = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        if (value_at<TPR, VEC>(c, t) < len)
#pragma unroll
            for (int j = 0; j < VEC; ++j) { const A d = x[c][j] - about; sq += d * d; }
    }
    sq = team_sum<(TPR < 32 ? TPR : 32)>(sq);
    if (TPR <= 32) {
        mean = about;
    } else {
        A* st = shared + (turn & 1) * 3 * WARPS;           // two sets: the next row's is written while this one is still read
        const int warp = t >> 5, lane = t & 31;
        if (lane == 0) { st[warp] = sum; st[WARPS + warp] = sq; st[2 * WARPS + warp] = (A)held; }
        __syncthreads();
        const A s = lane < WARPS ? st[lane] : (A)0, q = lane < WARPS ? st[WARPS + lane] : (A)0, h = lane < WARPS ? st[2 * WARPS + lane] : (A)0;
        mean = team_sum<32>(s) / (A)len;
        const A d = h > 0 ? s / h - mean : (A)0;
        sq = team_sum<32>(q + h * d * d);
    }
    rstd = inv_sqrt<A>(sq / (A)len + eps);
}

template <class X, int VEC, int TPR, int EPT, bool KEYED>
__global__ void __launch_bounds__(team_block(TPR)) norm_kernel(NormArgs a, View v)
{
    typedef typename Acc<X>::type A;
    constexpr int CH = EPT / VEC, TEAMS = team_block(TPR) / TPR;
    __shared__ A shared[TPR > 32 ? 6 * (TPR / 32) : 1];
    grid_dependency_wait();
    const int t = threadIdx.x % TPR, team = threadIdx.x / TPR;
    A w[CH][VEC], b[CH][VEC];
    load_params<X, A, VEC, TPR, CH>(a.w, a.w_type, a.w_vec, a.len, t, (A)1, w);
    load_params<X, A, VEC, TPR, CH>(a.b, a.w_type, a.w_vec, a.len, t, (A)0, b);
    int turn = 0;
    for (uint64_t base = (uint64_t)blockIdx.x * TEAMS; base < a.n; base += (uint64_t)gridDim.x * TEAMS, ++turn) {
        const uint64_t row = base + team;
        const bool in = row < a.n;
        const X* src = nullptr;
        const X* pend = nullptr;
        if (KEYED) {
            if (in) {
                const uint32_t key = __ldg(a.keys + row);
                if (key < v.num_keys) {
                    src = (const X*)v.val + (uint64_t)key * a.len;
                    if (key_is_hot(v, key)) {
                        const uint32_t slot = (uint32_t)__ldg(v.slot_of + key);
                        pend = (const X*)v.dval + ((uint64_t)worker_of_item(row, a.n, v.R) * v.Hcap + slot) * a.len;
                    }
                    if (v.count && t == 0) {
                        atomicAdd(v.cnt + key, 1ull);
                        atomicAdd(pend ? &v.st->hot_hits : &v.st->cold_hits, 1ull);
                    }
                } else if (t == 0) {
                    flag_bad_key(v);
                }
            }
        } else if (in) {
            src = (const X*)a.x + row * a.xs;
        }
        A x[CH][VEC];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const uint32_t at = value_at<TPR, VEC>(c, t);
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[c][j] = 0;
            if (src && at < a.len) {
                const Pack<X, VEC> r = load_pack<X, VEC>(src + at);
                unpack<A>(r, x[c]);
                if (KEYED && pend) {
                    A d[VEC];
                    unpack<A>(load_pack<X, VEC>(pend + at), d);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) x[c][j] += d[j];
                }
            }
        }
        if (KEYED && a.rows && in) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const uint32_t at = value_at<TPR, VEC>(c, t);
                if (at < a.len) store_values<X, VEC>((X*)a.rows + row * a.len + at, x[c]);
            }
        }
        A mean, rstd;
        row_stats<A, VEC, TPR, CH>(x, a.len, (A)a.eps, t, turn, shared, mean, rstd);
        if (!in) continue;
        if (t == 0) {
            if (a.mean) ((A*)a.mean)[row] = mean;
            if (a.rstd) ((A*)a.rstd)[row] = rstd;
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const uint32_t at = value_at<TPR, VEC>(c, t);
            if (at < a.len) {
                A y[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) y[j] = (x[c][j] - mean) * rstd * w[c][j] + b[c][j];
                store_chunk<X, A, VEC>(a.y, a.y_type, row * a.ys + at, y);
            }
        }
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

// Rows too long for registers: a block per row reads it three times, mostly from L2.
template <class X, int VEC, bool KEYED>
__global__ void __launch_bounds__(1024) norm_long_kernel(NormArgs a, View v)
{
    typedef typename Acc<X>::type A;
    __shared__ A shared[32];
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
        A sum = 0, sq = 0;
        for (uint32_t at = threadIdx.x * VEC; at < a.len; at += 1024 * VEC) {
            A x[VEC];
            read(at, x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) sum += x[j];
        }
        const A mean = block_sum(sum, shared) / (A)a.len;
        for (uint32_t at = threadIdx.x * VEC; at < a.len; at += 1024 * VEC) {
            A x[VEC];
            read(at, x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) sq += (x[j] - mean) * (x[j] - mean);
        }
        const A rstd = inv_sqrt<A>(block_sum(sq, shared) / (A)a.len + (A)a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) ((A*)a.mean)[row] = mean;
            if (a.rstd) ((A*)a.rstd)[row] = rstd;
        }
        for (uint32_t at = threadIdx.x * VEC; at < a.len; at += 1024 * VEC) {
            A x[VEC], w[1][VEC], b[1][VEC], y[VEC];
            read(at, x);
            if (KEYED && a.rows) store_values<X, VEC>((X*)a.rows + row * a.len + at, x);
            load_params<X, A, VEC, 1, 1>(a.w ? (const char*)a.w + (size_t)at * (sizeof(X) == 2 && a.w_type == NUPS_F32 ? 4 : sizeof(X)) : nullptr, a.w_type, a.w_vec, VEC, 0, (A)1, w);
            load_params<X, A, VEC, 1, 1>(a.b ? (const char*)a.b + (size_t)at * (sizeof(X) == 2 && a.w_type == NUPS_F32 ? 4 : sizeof(X)) : nullptr, a.w_type, a.w_vec, VEC, 0, (A)0, b);
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

template <class X, int VEC, bool KEYED>
nups_status launch_norm(nups_store* s, const NormArgs& a, const View& v, cudaStream_t st)
{
    const uint32_t len = a.len;
#define NUPS_NORM(TPR_, EPT_)                                                                                                              \
    {                                                                                                                                      \
        constexpr int TEAMS = team_block(TPR_) / TPR_;                                                                                     \
        static const unsigned resident = resident_blocks(norm_kernel<X, VEC, TPR_, EPT_, KEYED>, team_block(TPR_));                        \
        const unsigned grid = grid_for(a.n, TEAMS, (unsigned)s->sm_count * resident);                                                      \
        nups_launch_dependent(norm_kernel<X, VEC, TPR_, EPT_, KEYED>, grid, team_block(TPR_), 0, st, a, v);                                \
    }
    if (len <= 64) NUPS_NORM(8, 8)
    else if (len <= 128) NUPS_NORM(8, 16)
    else if (len <= 256) NUPS_NORM(32, 8)
    else if (len <= 512) NUPS_NORM(32, 16)
    else if (len <= 1024) NUPS_NORM(128, 8)
    else if (len <= 2048) NUPS_NORM(256, 8)
    else if (len <= 4096) NUPS_NORM(256, 16)
    else if (len <= 8192) NUPS_NORM(512, 16)
    else if (len <= 16384) NUPS_NORM(1024, 16)
    else nups_launch_dependent(norm_long_kernel<X, VEC, KEYED>, grid_for(a.n, 1, (unsigned)s->sm_count * 2), 1024, 0, st, a, v);
#undef NUPS_NORM
    LAUNCH_CHECK(s);
    return NUPS_OK;
}

bool aligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// weight and bias may be read VEC values at a time
int params_vec(const NormArgs& a, int x_type, int vec)
{
    const size_t run = (size_t)vec * (a.w_type == NUPS_F32 && x_type != NUPS_F64 ? 4 : type_bytes(x_type));
    const size_t need = run > 16 ? 16 : run;
    return aligned(a.w, need) && aligned(a.b, need);
}

bool w_type_fits(int x_type, int w_type) { return w_type == x_type || (w_type == NUPS_F32 && x_type != NUPS_F64); }
bool other_type_fits(int x_type, int t) { return t == x_type || (x_type == NUPS_F32 && (t == NUPS_F16 || t == NUPS_BF16)); }
bool eps_fits(int x_type, double eps) { return eps > 0 && eps < 1e30 && (x_type == NUPS_F64 || (float)eps > 0); }

// Do rows of `len` values of this type, `stride` apart, allow runs of `vec` values?
bool rows_allow(const void* p, int type, uint64_t stride, uint32_t len, int vec, uint64_t n)
{
    const size_t run = type_bytes(type) * vec, need = run > 16 ? 16 : run;
    return len % vec == 0 && aligned(p, need) && (n <= 1 || stride % vec == 0);
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
    nups_status rc = on_own_device(s);
    if (rc != NUPS_OK || n == 0) return rc;
    NormArgs a = {d_x, x_stride, d_y, y_stride, d_weight, d_bias, d_mean, d_rstd, n, len, y_type, w_type, 0, eps, nullptr, nullptr};
    const View v = {};
    cudaStream_t st = (cudaStream_t)stream;
    const int vec = (int)(16 / type_bytes(x_type));
    const bool wide = rows_allow(d_x, x_type, x_stride, len, vec, n) && rows_allow(d_y, y_type, y_stride, len, vec, n);
    a.w_vec = wide && params_vec(a, x_type, vec);
    switch (x_type) {
        case NUPS_F64: return wide ? launch_norm<double, 2, false>(s, a, v, st) : launch_norm<double, 1, false>(s, a, v, st);
        case NUPS_F32: return wide ? launch_norm<float, 4, false>(s, a, v, st) : launch_norm<float, 1, false>(s, a, v, st);
        case NUPS_F16: return wide ? launch_norm<__half, 8, false>(s, a, v, st) : launch_norm<__half, 1, false>(s, a, v, st);
        default: return wide ? launch_norm<__nv_bfloat16, 8, false>(s, a, v, st) : launch_norm<__nv_bfloat16, 1, false>(s, a, v, st);
    }
}

extern "C" nups_status nups_pull_norm(nups_store* s, const uint32_t* d_keys, uint64_t n, const void* d_weight, const void* d_bias, double eps,
                                      void* d_y, int y_type, void* d_rows, void* d_mean, void* d_rstd, void* stream)
{
    if (!s) return NUPS_EINVAL;
    const int type = s->vb == 8 ? NUPS_F64 : NUPS_F32;
    if (!other_type_fits(type, y_type) || !eps_fits(type, eps) || n >= (1ull << 32) || (n && (!d_keys || !d_y))) return NUPS_EINVAL;
    if (!aligned(d_y, 16) || !aligned(d_rows, 16)) return NUPS_EINVAL;
    nups_status rc = on_own_device(s);
    if (rc != NUPS_OK || n == 0) return rc;
    NormArgs a = {s->val, s->value_len, d_y, s->value_len, d_weight, d_bias, d_mean, d_rstd, n, s->value_len, y_type, type, 0, eps, d_keys, d_rows};
    a.w_vec = params_vec(a, type, type == NUPS_F64 ? 2 : 4);
    const View v = nups_view(s);
    return type == NUPS_F64 ? launch_norm<double, 2, true>(s, a, v, (cudaStream_t)stream) : launch_norm<float, 4, true>(s, a, v, (cudaStream_t)stream);
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
};

// One pass: a team holds x and dy of a row in registers and, over all of its rows, its columns' shares of dweight and dbias.
template <class X, int VEC, int TPR, int EPT>
__global__ void __launch_bounds__(team_block(TPR)) norm_grad_kernel(GradArgs a)
{
    typedef typename Acc<X>::type A;
    constexpr int CH = EPT / VEC, BLOCK = team_block(TPR), TEAMS = BLOCK / TPR, WARPS = BLOCK / 32;
    __shared__ A shared[TPR > 32 ? 4 * WARPS : WARPS * TPR * EPT];
    grid_dependency_wait();
    const int t = threadIdx.x % TPR, team = threadIdx.x / TPR;
    A w[CH][VEC], dw[CH][VEC], db[CH][VEC];
    load_params<X, A, VEC, TPR, CH>(a.w, a.w_type, a.w_vec, a.len, t, (A)1, w);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < VEC; ++j) dw[c][j] = db[c][j] = 0;
    int turn = 0;
    const A inv_len = (A)1 / (A)a.len;
    for (uint64_t base = (uint64_t)blockIdx.x * TEAMS; base < a.n; base += (uint64_t)gridDim.x * TEAMS, ++turn) {
        const uint64_t row = base + team;
        const bool in = row < a.n;
        const A mean = in ? ((const A*)a.mean)[row] : (A)0, rstd = in ? ((const A*)a.rstd)[row] : (A)0;
        A h[CH][VEC], g[CH][VEC];
        A s1 = 0, s2 = 0;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const uint32_t at = value_at<TPR, VEC>(c, t);
#pragma unroll
            for (int j = 0; j < VEC; ++j) h[c][j] = g[c][j] = 0;
            if (in && at < a.len) {
                unpack<A>(load_pack<X, VEC>((const X*)a.x + row * a.xs + at), h[c]);
                load_chunk<X, A, VEC>(a.dy, a.dy_type, row * a.dys + at, g[c]);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    h[c][j] = (h[c][j] - mean) * rstd;
                    dw[c][j] += g[c][j] * h[c][j];
                    db[c][j] += g[c][j];
                    g[c][j] *= w[c][j];
                    s1 += g[c][j];
                    s2 += g[c][j] * h[c][j];
                }
            }
        }
        if (!a.dx) continue;                                // the same for the whole grid
        s1 = team_sum<(TPR < 32 ? TPR : 32)>(s1);
        s2 = team_sum<(TPR < 32 ? TPR : 32)>(s2);
        if (TPR > 32) {
            A* st = shared + (turn & 1) * 2 * WARPS;
            const int lane = t & 31;
            if (lane == 0) { st[t >> 5] = s1; st[WARPS + (t >> 5)] = s2; }
            __syncthreads();
            s1 = team_sum<32>(lane < WARPS ? st[lane] : (A)0);
            s2 = team_sum<32>(lane < WARPS ? st[WARPS + lane] : (A)0);
        }
        s1 *= inv_len;
        s2 *= inv_len;
        if (!in) continue;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const uint32_t at = value_at<TPR, VEC>(c, t);
            if (at < a.len) {
                A d[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) d[j] = (g[c][j] - s1 - h[c][j] * s2) * rstd;
                store_values<X, VEC>((X*)a.dx + row * a.dxs + at, d);
            }
        }
    }
    if (!a.part) return;
    A* out = (A*)a.part + (uint64_t)blockIdx.x * 2 * a.len;
    if (TPR > 32) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const uint32_t at = value_at<TPR, VEC>(c, t);
            if (at < a.len)
#pragma unroll
                for (int j = 0; j < VEC; ++j) { out[at + j] = dw[c][j]; out[a.len + at + j] = db[c][j]; }
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
                }
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < a.len; i += BLOCK) {
                A sum = 0;
#pragma unroll
                for (int k = 0; k < WARPS; ++k) sum += shared[k * TPR * EPT + i];
                out[which * a.len + i] = sum;
            }
        }
    }
}

// Rows too long for registers, first pass: a block per row leaves mean(g) and mean(g h).
template <class X, int VEC>
__global__ void __launch_bounds__(1024) norm_grad_sums_kernel(GradArgs a, typename Acc<X>::type* sums)
{
    typedef typename Acc<X>::type A;
    __shared__ A shared[32];
    grid_dependency_wait();
    for (uint64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const A mean = ((const A*)a.mean)[row], rstd = ((const A*)a.rstd)[row];
        A s1 = 0, s2 = 0;
        for (uint32_t at = threadIdx.x * VEC; at < a.len; at += 1024 * VEC) {
            A x[VEC], g[VEC], w[1][VEC];
            unpack<A>(load_pack<X, VEC>((const X*)a.x + row * a.xs + at), x);
            load_chunk<X, A, VEC>(a.dy, a.dy_type, row * a.dys + at, g);
            load_params<X, A, VEC, 1, 1>(a.w ? (const char*)a.w + (size_t)at * (sizeof(X) == 2 && a.w_type == NUPS_F32 ? 4 : sizeof(X)) : nullptr, a.w_type, a.w_vec, VEC, 0, (A)1, w);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const A gj = g[j] * w[0][j];
                s1 += gj;
                s2 += gj * ((x[j] - mean) * rstd);
            }
        }
        s1 = block_sum(s1, shared);
        s2 = block_sum(s2, shared);
        if (threadIdx.x == 0) { sums[2 * row] = s1 / (A)a.len; sums[2 * row + 1] = s2 / (A)a.len; }
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
    load_params<X, A, VEC, 1, 1>(a.w ? (const char*)a.w + (size_t)at * (sizeof(X) == 2 && a.w_type == NUPS_F32 ? 4 : sizeof(X)) : nullptr, a.w_type, a.w_vec, VEC, 0, (A)1, w);
#pragma unroll
    for (int j = 0; j < VEC; ++j) dw[j] = db[j] = 0;
    for (uint64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
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
    if (a.part) {
        A* out = (A*)a.part + (uint64_t)blockIdx.y * 2 * a.len + at;
#pragma unroll
        for (int j = 0; j < VEC; ++j) { out[j] = dw[j]; out[a.len + j] = db[j]; }
    }
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

constexpr uint32_t GRAD_LONG = 8192;       // longer rows (fp64: half of it) take two passes
uint32_t grad_long_from(int type) { return type == NUPS_F64 ? GRAD_LONG / 2 : GRAD_LONG; }

// Blocks that leave sums: a rule on the sizes alone, so that the order of the additions is theirs too.
uint32_t grad_teams(uint32_t len) { return len <= 128 ? 32 : len <= 512 ? 8 : 1; }
unsigned grad_blocks(const nups_store* s, uint64_t n, uint32_t len, int type)
{
    const unsigned sm = (unsigned)s->sm_count;
    if (len > grad_long_from(type)) return grid_for(n, 16, 32);
    return grid_for(n, grad_teams(len), sm * (len <= 512 ? 4 : len <= 2048 ? 6 : len <= 4096 ? 2 : 1));
}
uint64_t grad_part_bytes(const nups_store* s, uint64_t n, uint32_t len, int type)
{
    return (uint64_t)grad_blocks(s, n, len, type) * 2 * len * (type == NUPS_F64 ? 8 : 4);
}

template <class X, int VEC>
nups_status launch_grad(nups_store* s, GradArgs a, int x_type, void* d_dw, void* d_db, char* scratch, cudaStream_t st)
{
    typedef typename Acc<X>::type A;
    const uint32_t len = a.len;
    const unsigned blocks = grad_blocks(s, a.n, len, x_type);
#define NUPS_GRAD(TPR_, EPT_) nups_launch_dependent(norm_grad_kernel<X, VEC, TPR_, EPT_>, blocks, team_block(TPR_), 0, st, a)
    if (len > grad_long_from(x_type)) {
        A* sums = (A*)(scratch + (a.part ? (grad_part_bytes(s, a.n, len, x_type) + 255) / 256 * 256 : 0));
        if (a.dx) {
            nups_launch_dependent(norm_grad_sums_kernel<X, VEC>, grid_for(a.n, 1, (unsigned)s->sm_count * 2), 1024, 0, st, a, sums);
            LAUNCH_CHECK(s);
        }
        nups_launch_dependent(norm_grad_apply_kernel<X, VEC>, dim3(grid_for(len, 256 * VEC), blocks), 256, 0, st, a, (const A*)sums);
    }
    else if (len <= 64) NUPS_GRAD(8, 8);
    else if (len <= 128) NUPS_GRAD(8, 16);
    else if (len <= 256) NUPS_GRAD(32, 8);
    else if (len <= 512) NUPS_GRAD(32, 16);
    else if (len <= 1024) NUPS_GRAD(128, 8);
    else if (len <= 2048) NUPS_GRAD(128, 16);
    else if (len <= 4096) NUPS_GRAD(256, 16);
    else NUPS_GRAD(512, 16);
#undef NUPS_GRAD
    LAUNCH_CHECK(s);
    if (a.part) {
        const dim3 grid((len + 31) / 32, 2);
        if (sizeof(X) == 2 && a.w_type == NUPS_F32) nups_launch_dependent(norm_grad_join_kernel<A, float>, grid, 1024, 0, st, (const A*)a.part, blocks, len, (float*)d_dw, (float*)d_db);
        else nups_launch_dependent(norm_grad_join_kernel<A, X>, grid, 1024, 0, st, (const A*)a.part, blocks, len, (X*)d_dw, (X*)d_db);
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
    const bool sums = d_dweight || d_dbias;
    const bool needs = n && (sums || (d_dx && len > grad_long_from(x_type)));
    uint64_t bytes = 0;
    nups_layer_norm_grad_scratch(s, n, len, x_type, &bytes);
    if (needs && (!d_scratch || scratch_bytes < bytes || !aligned(d_scratch, 256))) return NUPS_EINVAL;
    nups_status rc = on_own_device(s);
    if (rc != NUPS_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    if (n == 0) {
        if (d_dweight) CK(cudaMemsetAsync(d_dweight, 0, (size_t)len * type_bytes(w_type), st));
        if (d_dbias) CK(cudaMemsetAsync(d_dbias, 0, (size_t)len * type_bytes(w_type), st));
        return NUPS_OK;
    }
    if (!sums && !d_dx) return NUPS_OK;
    GradArgs a = {d_x, x_stride, d_dy, dy_stride, d_mean, d_rstd, d_weight, d_dx, dx_stride, sums ? d_scratch : nullptr, n, len, dy_type, w_type, 0};
    const int vec = (int)(16 / type_bytes(x_type));
    const bool wide = rows_allow(d_x, x_type, x_stride, len, vec, n) && rows_allow(d_dy, dy_type, dy_stride, len, vec, n) &&
                      (!d_dx || rows_allow(d_dx, x_type, dx_stride, len, vec, n));
    const size_t run = (size_t)vec * (w_type == NUPS_F32 && x_type != NUPS_F64 ? 4 : type_bytes(x_type));
    a.w_vec = wide && aligned(d_weight, run > 16 ? 16 : run);
    char* scratch = (char*)d_scratch;
    switch (x_type) {
        case NUPS_F64: return wide ? launch_grad<double, 2>(s, a, x_type, d_dweight, d_dbias, scratch, st) : launch_grad<double, 1>(s, a, x_type, d_dweight, d_dbias, scratch, st);
        case NUPS_F32: return wide ? launch_grad<float, 4>(s, a, x_type, d_dweight, d_dbias, scratch, st) : launch_grad<float, 1>(s, a, x_type, d_dweight, d_dbias, scratch, st);
        case NUPS_F16: return wide ? launch_grad<__half, 8>(s, a, x_type, d_dweight, d_dbias, scratch, st) : launch_grad<__half, 1>(s, a, x_type, d_dweight, d_dbias, scratch, st);
        default: return wide ? launch_grad<__nv_bfloat16, 8>(s, a, x_type, d_dweight, d_dbias, scratch, st) : launch_grad<__nv_bfloat16, 1>(s, a, x_type, d_dweight, d_dbias, scratch, st);
    }
}
