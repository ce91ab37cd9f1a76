// A router over experts: softmax and choice of the largest logits per item, counts per expert, balance and z losses, and the
// gradient of the logits.
//
// One pass over the logits per direction.  An item's logits are held in the registers of a team of TPR lanes (EPT each; few lanes
// with many logits, so that what the team does together is shared by several items of a warp).  The choice takes one reduction over
// the team per chosen expert: each lane keeps its KEPT largest logits as whole numbers in the order of the logits (for 16-bit types
// with the expert's number in the bits that the logit leaves free, so that equal logits are told apart by the same comparison), and
// looks through its logits again only when all of those were chosen.  The sums over items (P, lse^2) stay in registers until the
// block ends; the four blocks of a cluster add theirs through shared memory and leave them in scratch, and a last small kernel
// adds the clusters' in order.
#include <atomic>
#include <cooperative_groups.h>
#include <math.h>
#include <math_constants.h>

#include "nups_types.cuh"

namespace {

struct RouteArgs {
    const void* logits;
    uint64_t stride, n;
    uint32_t experts, top;
    const uint8_t* active;
    int renormalize, sums;     // sums: P and Z are wanted
    float balance, z;
    int32_t* choice;
    float *weight, *lse;
    uint64_t *counts, *tokens;
    float *prob, *loss;
    float* part_p;             // [blocks][experts], then [blocks] sums of lse^2
    uint32_t* part_c;          // [blocks][experts] counts, then [blocks] items
};

constexpr int ROUTE_BLOCK = 256, ROUTE_CLUSTER = 4;
__host__ __device__ constexpr int route_slots(int tpr) { return tpr == 32 ? 1 : 4; }      // chosen experts that a lane keeps

template <int TPR> __device__ __forceinline__ float lanes_sum(float x)
{
#pragma unroll
    for (int o = TPR / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}
template <int TPR> __device__ __forceinline__ float lanes_most(float x)
{
#pragma unroll
    for (int o = TPR / 2; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
    return x;
}
template <int TPR> __device__ __forceinline__ uint32_t lanes_max(uint32_t x)
{
    if constexpr (TPR == 32) {
        return __reduce_max_sync(0xFFFFFFFFu, x);
    } else {
#pragma unroll
        for (int o = TPR / 2; o > 0; o >>= 1) x = max(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
        return x;
    }
}
template <int TPR> __device__ __forceinline__ uint32_t lanes_min(uint32_t x)
{
    if constexpr (TPR == 32) {
        return __reduce_min_sync(0xFFFFFFFFu, x);
    } else {
#pragma unroll
        for (int o = TPR / 2; o > 0; o >>= 1) x = min(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
        return x;
    }
}

// Whole numbers in the order of the logits; up to NONE = never chosen (-infinity).  -0 counts as +0; x is not NaN.
constexpr uint32_t NONE = 0x007FFFFFu;
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u); }
// fp16 and bf16 leave at least 13 bits of a float's mantissa free: the larger number there is the lower expert
constexpr uint32_t FREE = 0x1FFFu;
// tag = 0x80000000 | (FREE - e): the free bits of x are zero, so the key is two operations on the number's bits
__device__ __forceinline__ uint32_t ordered_with(float x, uint32_t tag)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) & (0x7FFFFFFFu & ~FREE)) ^ tag;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return from_ordered(key & 0x80000000u ? key & ~FREE : key | FREE); }

// The largest keys of a lane, in order, each with its expert (PACKED: in the key).
template <bool PACKED, int KEPT> struct Largest {
    uint32_t key[KEPT], expert[PACKED ? 1 : KEPT];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < KEPT; ++i) key[i] = 0;
    }
    __device__ __forceinline__ void take(uint32_t k, uint32_t e)
    {
        if constexpr (PACKED) {
#pragma unroll
            for (int i = 0; i < KEPT; ++i) {
                const uint32_t more = max(key[i], k);
                k = min(key[i], k);
                key[i] = more;
            }
        } else {                                            // experts come in ascending order: an equal key stays behind
            bool more = false;
#pragma unroll
            for (int i = 0; i < KEPT; ++i) {
                more = more || k > key[i];                  // what is behind its place moves down, equal or not
                const uint32_t tk = more ? key[i] : k, te = more ? expert[i] : e;
                key[i] = more ? k : key[i];
                expert[i] = more ? e : expert[i];
                k = tk;
                e = te;
            }
        }
    }
    __device__ __forceinline__ void drop()
    {
#pragma unroll
        for (int i = 0; i + 1 < KEPT; ++i) {
            key[i] = key[i + 1];
            if constexpr (!PACKED) expert[i] = expert[i + 1];
        }
        key[KEPT - 1] = 0;
    }
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

template <int TPR, int VEC> __device__ __forceinline__ uint32_t expert_at(int i, int t)
{
    return (uint32_t)(((i / VEC) * TPR + t) * VEC + i % VEC);
}

// A lane's logits as they lie in memory, and as floats (-infinity where there is none).
template <class X, int VEC, int TPR, int EPT>
__device__ __forceinline__ void fetch_logits(const X* row, bool in, uint32_t experts, int t, Pack<X, VEC> (&raw)[EPT / VEC])
{
#pragma unroll
    for (int c = 0; c < EPT / VEC; ++c)
        if (in && expert_at<TPR, VEC>(c * VEC, t) < experts) raw[c] = load_pack<X, VEC>(row + expert_at<TPR, VEC>(c * VEC, t));
}
template <class X, int VEC, int TPR, int EPT>
__device__ __forceinline__ void read_logits(const Pack<X, VEC> (&raw)[EPT / VEC], bool in, uint32_t experts, int t, float (&x)[EPT])
{
#pragma unroll
    for (int c = 0; c < EPT / VEC; ++c) {
        if (in && expert_at<TPR, VEC>(c * VEC, t) < experts) unpack<float>(raw[c], x + c * VEC);
        else
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[c * VEC + j] = -CUDART_INF_F;
    }
}

// Counts and mean of one expert; returns its share of B's sum.
__device__ __forceinline__ float finish_expert(const RouteArgs& a, uint32_t e, float p, uint32_t c, float T)
{
    const float P = p / T;
    a.counts[e] = c;
    if (a.prob) a.prob[e] = P;
    return (float)c * P;
}
// What is left when B's sum is known; one thread.
__device__ __forceinline__ void finish_losses(const RouteArgs& a, float b, float z, uint32_t tokens, float T)
{
    *a.tokens = tokens;
    if (!a.loss) return;
    const float B = b * ((float)a.experts / ((float)a.top * T)), Z = z / T;
    a.loss[0] = a.balance * B + a.z * Z;
    a.loss[1] = B;
    a.loss[2] = Z;
}

// e^(x - most), elementwise
template <int EPT> __device__ __forceinline__ void exponentials(const float* x, float most, float* ex)
{
    const float minus = -most, log2e = 1.4426950408889634f;
    run_add<EPT, true>(ex, x, &minus);
    run_scale<EPT>(ex, ex, log2e);
#pragma unroll
    for (int i = 0; i < EPT; ++i) ex[i] = exp2_fast(ex[i]);
}

// Blocks per multiprocessor as in route_blocks.  With 16 or 32 logits per lane that leaves too few registers: by 16-byte loads, 12 to 44
// bytes a thread are spilled with 32 16-bit logits, 28 to 180 with 16 float ones.
template <class X, int VEC, int TPR, int EPT, int KEPT>
__global__ void __launch_bounds__(ROUTE_BLOCK, EPT <= 8 ? 4 : EPT <= 16 ? 3 : 2) route_kernel(RouteArgs a)
{
    constexpr int TEAMS = ROUTE_BLOCK / TPR, CAP = TPR * EPT, SLOTS = route_slots(TPR), WARPS = ROUTE_BLOCK / 32;
    constexpr bool PACKED = sizeof(X) == 2;
    __shared__ uint32_t chosen[CAP];                        // counts of this block
    __shared__ float sums[WARPS][CAP > 512 ? 512 : CAP];
    __shared__ float psum[CAP];
    __shared__ float zsum[WARPS], bsum[WARPS];
    __shared__ uint32_t tsum[WARPS];
    __shared__ float z_block;
    __shared__ uint32_t t_block;
    for (int e = threadIdx.x; e < CAP; e += ROUTE_BLOCK) chosen[e] = 0;
    __syncthreads();
    grid_dependency_wait();
    const int t = threadIdx.x % TPR, team = threadIdx.x / TPR;
    float acc[EPT], zacc = 0;
    uint32_t items = 0;
#pragma unroll
    for (int i = 0; i < EPT; ++i) acc[i] = 0;
    const uint64_t step = (uint64_t)gridDim.x * TEAMS;
    uint64_t row = (uint64_t)blockIdx.x * TEAMS + team;
    const uint32_t tag = 0x80000000u | (FREE ^ (uint32_t)(t * VEC));      // of the lane's first expert; the others differ in other bits
    for (uint64_t base = (uint64_t)blockIdx.x * TEAMS; base < a.n; base += step, row += step) {
        const bool in = row < a.n;
        bool on = in && (!a.active || a.active[row]);
        float x[EPT], total, most;                          // logits, then their exponentials
        Pack<X, VEC> raw[EPT / VEC];
        fetch_logits<X, VEC, TPR, EPT>((const X*)a.logits + row * a.stride, in, a.experts, t, raw);       // does not wait for the mask
        read_logits<X, VEC, TPR, EPT>(raw, on, a.experts, t, x);
        uint32_t slot_u[SLOTS];
        int32_t slot_e[SLOTS];
        bool any, nan_item = false;
        auto key_of = [&](int i) { return PACKED ? ordered_with(x[i], tag ^ expert_at<TPR, VEC>(i, 0)) : ordered(x[i]); };
        for (int pass = 0;; ++pass) {
            Largest<PACKED, KEPT> top;
            int left = 0;                                   // of those kept
            uint32_t u = 0xFFFFFFFFu, e = 0;                // the last one chosen
            most = 0.0f;
            any = false;
#pragma unroll
            for (int s = 0; s < SLOTS; ++s) {
                slot_u[s] = 0;
                slot_e[s] = -1;
                if (s * TPR >= (int)a.top) continue;
                for (int l = 0; l < TPR; ++l) {
                    if (s * TPR + l >= (int)a.top) break;
                    if (left == 0) {                        // none are kept (any more): the largest after u
                        left = KEPT;
                        top.clear();
#pragma unroll
                        for (int i = 0; i < EPT; ++i) {
                            const uint32_t w = key_of(i), ei = expert_at<TPR, VEC>(i, t);
                            top.take(w < u || (!PACKED && w == u && ei > e) ? w : 0u, ei);
                        }
                    }
                    u = lanes_max<TPR>(top.key[0]);
                    if constexpr (PACKED) e = FREE - (u & FREE);
                    else e = lanes_min<TPR>(top.key[0] == u ? top.expert[0] : 0xFFFFFFFFu);
                    bool mine = top.key[0] == u;
                    if constexpr (!PACKED) mine = mine && top.expert[0] == e;
                    if (mine) {
                        top.drop();
                        --left;
                    }
                    const bool some = u > (PACKED ? NONE | FREE : NONE);
                    if (s == 0 && l == 0) {
                        any = some;
                        most = any ? (PACKED ? logit_of(u) : from_ordered(u)) : 0.0f;
                    }
                    if (t == l && some) { slot_u[s] = u; slot_e[s] = (int32_t)e; }
                }
            }
            exponentials<EPT>(x, most, x);
            float two_sums[2] = {0, 0};
            sum_run<EPT>(two_sums, x);
            total = lanes_sum<TPR>(two_sums[0] + two_sums[1]);
            if (pass == 1) {
                if (nan_item) total = CUDART_NAN_F;
                break;
            }
            nan_item = total != total;
            if (!__any_sync(0xFFFFFFFFu, nan_item)) break;
            // NaN, which the order above knows nothing of (or +infinity): once more with NaN as what is not chosen; the item's
            // sum stays NaN
            fetch_logits<X, VEC, TPR, EPT>((const X*)a.logits + row * a.stride, on, a.experts, t, raw);
            read_logits<X, VEC, TPR, EPT>(raw, on, a.experts, t, x);
#pragma unroll
            for (int i = 0; i < EPT; ++i)
                if (x[i] != x[i]) x[i] = -CUDART_INF_F;
        }
        if (!any && total == 0.0f) on = false;              // nothing but -infinity
        const float inv = on ? 1.0f / total : 0.0f;
        float kept[SLOTS], kept_sum = 0;
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            kept[s] = slot_e[s] >= 0 ? exp2_fast(((PACKED ? logit_of(slot_u[s]) : from_ordered(slot_u[s])) - most) * 1.4426950408889634f) : 0.0f;
            kept_sum += kept[s];
        }
        float scale = inv;
        if (a.renormalize) {
            kept_sum = lanes_sum<TPR>(kept_sum);
            scale = kept_sum != 0.0f ? 1.0f / kept_sum : 0.0f;
            if (total != total) scale = total;
        }
        if (in) {
#pragma unroll
            for (int s = 0; s < SLOTS; ++s) {
                const uint32_t j = s * TPR + t;
                if (j < a.top) {
                    a.choice[row * a.top + j] = slot_e[s];
                    a.weight[row * a.top + j] = slot_e[s] >= 0 ? kept[s] * scale : 0.0f;
                    if (slot_e[s] >= 0) atomicAdd(&chosen[slot_e[s]], 1u);
                }
            }
        }
        if (on) {
            const float lse = most + logf(total);
            if (t == 0) {
                if (a.lse) a.lse[row] = lse;
                zacc += lse * lse;
                ++items;
            }
            if (a.sums) run_fma<EPT, false, true, false>(acc, x, &inv, acc);
        } else if (in && t == 0 && a.lse) {
            a.lse[row] = 0.0f;
        }
    }
    // the block's sums: teams of a warp by shuffles, warps through shared memory
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 16; o >= TPR; o >>= 1)
#pragma unroll
        for (int i = 0; i < EPT; ++i) acc[i] += __shfl_xor_sync(0xFFFFFFFFu, acc[i], o);
    zacc = lanes_sum<32>(zacc);
    items = __reduce_add_sync(0xFFFFFFFFu, items);
    if (lane == 0) { zsum[warp] = zacc; tsum[warp] = items; }
    __syncthreads();
    float z = 0;
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) { z += zsum[w]; m += tsum[w]; }
    constexpr int PART = CAP > 512 ? 512 : CAP;             // experts per round
#pragma unroll
    for (int r = 0; r < CAP / PART; ++r) {
        __syncthreads();
        if (lane < TPR)
#pragma unroll
            for (int i = 0; i < EPT; ++i) {
                const uint32_t e = expert_at<TPR, VEC>(i, t);
                if (e / PART == r) sums[warp][e % PART] = acc[i];
            }
        __syncthreads();
        for (int k = threadIdx.x; k < PART; k += ROUTE_BLOCK) {
            float p = 0;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) p += sums[w][k];
            psum[r * PART + k] = p;
        }
    }
    if (threadIdx.x == 0) { z_block = z; t_block = m; }
    __syncthreads();
    if (gridDim.x == 1) {                                   // this block's sums are the call's
        const float T = m ? (float)m : 1.0f;
        float b = 0;
        for (uint32_t e = threadIdx.x; e < a.experts; e += ROUTE_BLOCK) b += finish_expert(a, e, psum[e], chosen[e], T);
        b = lanes_sum<32>(b);
        if (lane == 0) bsum[warp] = b;
        __syncthreads();
        if (threadIdx.x == 0) {
            b = 0;
            for (int w = 0; w < WARPS; ++w) b += bsum[w];
            finish_losses(a, b, z, m, T);
        }
        return;
    }
    // the cluster's sums, each block a fourth of the experts
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    cluster.sync();
    const uint32_t rank = cluster.block_rank(), group = blockIdx.x / ROUTE_CLUSTER, groups = gridDim.x / ROUTE_CLUSTER;
    for (uint32_t e = rank + ROUTE_CLUSTER * threadIdx.x; e < a.experts; e += ROUTE_CLUSTER * ROUTE_BLOCK) {
        float p = 0;
        uint32_t c = 0;
#pragma unroll
        for (int r = 0; r < ROUTE_CLUSTER; ++r) {
            p += *cluster.map_shared_rank(&psum[e], r);
            c += *cluster.map_shared_rank(&chosen[e], r);
        }
        a.part_p[(uint64_t)group * a.experts + e] = p;
        a.part_c[(uint64_t)group * a.experts + e] = c;
    }
    if (rank == 0 && threadIdx.x == 0) {
        z = 0;
        m = 0;
        for (int r = 0; r < ROUTE_CLUSTER; ++r) { z += *cluster.map_shared_rank(&z_block, r); m += *cluster.map_shared_rank(&t_block, r); }
        a.part_p[(uint64_t)groups * a.experts + group] = z;
        a.part_c[(uint64_t)groups * a.experts + group] = m;
    }
    cluster.sync();                                         // the blocks' shared memory stays until it was read
}

constexpr int JOIN_BLOCK = 1024, JOIN_CLUSTER = 8;
// The sums of all clusters: a cluster whose blocks take `width` experts each, JOIN_BLOCK / width threads per expert.
__global__ void __cluster_dims__(JOIN_CLUSTER) __launch_bounds__(JOIN_BLOCK) route_join_kernel(RouteArgs a, uint32_t blocks, uint32_t width)
{
    __shared__ float sp[JOIN_BLOCK];
    __shared__ uint32_t sc[JOIN_BLOCK];
    __shared__ float shared[32];
    __shared__ uint32_t shared_t[32];
    __shared__ float share;                                 // this block's part of B's sum
    grid_dependency_wait();
    const uint32_t run = threadIdx.x / width, runs = JOIN_BLOCK / width, e = blockIdx.x * width + threadIdx.x % width;
    float p = 0;
    uint32_t c = 0;
    if (e < a.experts)
#pragma unroll 8
        for (uint32_t b = run; b < blocks; b += runs) {
            p += __ldcg(a.part_p + (uint64_t)b * a.experts + e);
            c += __ldcg(a.part_c + (uint64_t)b * a.experts + e);
        }
    float z = 0;
    uint32_t m = 0;
    for (uint32_t b = threadIdx.x; b < blocks; b += JOIN_BLOCK) {
        z += __ldcg(a.part_p + (uint64_t)blocks * a.experts + b);
        m += __ldcg(a.part_c + (uint64_t)blocks * a.experts + b);
    }
    z = lanes_sum<32>(z);
    m = __reduce_add_sync(0xFFFFFFFFu, m);
    if ((threadIdx.x & 31) == 0) { shared[threadIdx.x >> 5] = z; shared_t[threadIdx.x >> 5] = m; }
    sp[threadIdx.x] = p;
    sc[threadIdx.x] = c;
    __syncthreads();
    z = lanes_sum<32>(shared[threadIdx.x & 31]);
    m = __reduce_add_sync(0xFFFFFFFFu, shared_t[threadIdx.x & 31]);
    for (uint32_t half = runs / 2; half > 0; half /= 2) {   // a tree over the runs
        if (run < half) {
            sp[threadIdx.x] += sp[threadIdx.x + half * width];
            sc[threadIdx.x] += sc[threadIdx.x + half * width];
        }
        __syncthreads();
    }
    const float T = m ? (float)m : 1.0f;
    float b = run == 0 && e < a.experts ? finish_expert(a, e, sp[threadIdx.x], sc[threadIdx.x], T) : 0.0f;
    b = lanes_sum<32>(b);
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = b;
    __syncthreads();
    if (threadIdx.x < 32) {
        b = lanes_sum<32>(shared[threadIdx.x]);
        if (threadIdx.x == 0) share = b;
    }
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    cluster.sync();
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        b = 0;
        for (unsigned r = 0; r < JOIN_CLUSTER; ++r) b += *cluster.map_shared_rank(&share, r);
        finish_losses(a, b, z, m, T);
    }
    cluster.sync();                                         // the blocks' shared memory stays until it was read
}

struct RouteGradArgs {
    const void* logits;
    uint64_t stride, n;
    uint32_t experts, top;
    const uint8_t* active;
    int renormalize;
    float balance, z;
    const int32_t* choice;
    const float *weight, *lse;
    const uint64_t *counts, *tokens;
    const float *dloss, *dweight;
    void* dlogits;
    uint64_t dstride;
};

// d_e = p_e (g_e - sum g p + 2 z dloss lse / T), g_e = balance dloss f_e / T (+ dweight where e was chosen); with renormalized
// weights the choices add w (dweight - sum dweight w) instead.  What the choices add is left in the team's row of shared memory
// by the lanes that hold them and picked up by the lanes that hold the logits.
template <class X, int VEC, int TPR, int EPT>
__global__ void __launch_bounds__(ROUTE_BLOCK) route_grad_kernel(RouteGradArgs a)
{
    constexpr int TEAMS = ROUTE_BLOCK / TPR, CAP = TPR * EPT, SLOTS = route_slots(TPR);
    __shared__ float extra[TEAMS][CAP];
    const int t = threadIdx.x % TPR, team = threadIdx.x / TPR;
    for (int e = t; e < CAP; e += TPR) extra[team][e] = 0.0f;
    grid_dependency_wait();
    const uint64_t tokens = *a.tokens;
    const float T = tokens ? (float)tokens : 1.0f;
    const float dloss = a.dloss ? *a.dloss : 1.0f;
    const float zf = dloss * a.z * 2.0f / T, bf = dloss * a.balance / T * ((float)a.experts / ((float)a.top * T));
    float g[EPT];
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
        const uint32_t e = expert_at<TPR, VEC>(i, t);
        g[i] = e < a.experts ? bf * (float)a.counts[e] : 0.0f;
    }
    __syncwarp();
    const uint64_t step = (uint64_t)gridDim.x * TEAMS;
    uint64_t row = (uint64_t)blockIdx.x * TEAMS + team;
    for (uint64_t base = (uint64_t)blockIdx.x * TEAMS; base < a.n; base += step, row += step) {
        const bool in = row < a.n, on = in && (!a.active || a.active[row]);
        Pack<X, VEC> raw[EPT / VEC];
        fetch_logits<X, VEC, TPR, EPT>((const X*)a.logits + row * a.stride, in, a.experts, t, raw);       // nothing waits for the mask
        const float lse = in ? a.lse[row] : 0.0f;
        int32_t c[SLOTS];
        float add[SLOTS], dw[SLOTS], part = 0;
        if (a.dweight) {
#pragma unroll
            for (int s = 0; s < SLOTS; ++s) {
                const uint32_t j = s * TPR + t;
                const bool has = in && j < a.top;
                c[s] = has ? a.choice[row * a.top + j] : -1;
                add[s] = has ? a.weight[row * a.top + j] : 0.0f;
                dw[s] = has ? a.dweight[row * a.top + j] : 0.0f;
            }
#pragma unroll
            for (int s = 0; s < SLOTS; ++s) {
                if (!on || (uint32_t)c[s] >= a.experts) { c[s] = -1; add[s] = dw[s] = 0.0f; }
                part += dw[s] * add[s];
            }
            if (a.renormalize) {                            // w (dweight - sum dweight w)
                const float mean = lanes_sum<TPR>(part);
                part = 0.0f;
#pragma unroll
                for (int s = 0; s < SLOTS; ++s) add[s] *= dw[s] - mean;
            } else {                                        // p dweight; the sum takes part in sum g p
#pragma unroll
                for (int s = 0; s < SLOTS; ++s) add[s] *= dw[s];
            }
#pragma unroll
            for (int s = 0; s < SLOTS; ++s)
                if (c[s] >= 0) atomicAdd(&extra[team][c[s]], add[s]);
            __syncwarp();
        }
        float p[EPT];                                       // logits, then probabilities
        read_logits<X, VEC, TPR, EPT>(raw, on, a.experts, t, p);
        // p about the largest logit, as forward: lse is rounded at its own size, and e^(logit - lse) would carry that rounding in every p
        float most = -CUDART_INF_F, two_sums[2] = {0, 0}, along[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < EPT; ++i) most = fmaxf(most, p[i]);             // passes over NaN, which the sum shows
        most = lanes_most<TPR>(most);
        exponentials<EPT>(p, most == -CUDART_INF_F ? 0.0f : most, p);
        sum_run<EPT>(two_sums, p);
        const float total = lanes_sum<TPR>(two_sums[0] + two_sums[1]);
        run_scale<EPT>(p, p, total == 0.0f ? 0.0f : 1.0f / total);          // 0: nothing but -infinity
        sum_run_of_products<EPT>(along, p, g);
        part += along[0] + along[1];
        const float off = zf * lse - lanes_sum<TPR>(part);
        if (in) {
#pragma unroll
            for (int k = 0; k < EPT / VEC; ++k) {
                const uint32_t e = expert_at<TPR, VEC>(k * VEC, t);
                if (e < a.experts) {
                    float d[VEC], more[VEC];
#pragma unroll
                    for (int j = 0; j < VEC; ++j) more[j] = a.dweight ? extra[team][e + j] : 0.0f;
                    run_add<VEC, true>(d, g + k * VEC, &off);
                    run_fma<VEC, false, false, false>(d, d, p + k * VEC, more);
                    if (!on)
#pragma unroll
                        for (int j = 0; j < VEC; ++j) d[j] = 0.0f;
                    store_values<X, VEC>((X*)a.dlogits + row * a.dstride + e, d);
                }
            }
        }
        if (a.dweight) {
            __syncwarp();
#pragma unroll
            for (int s = 0; s < SLOTS; ++s)
                if (c[s] >= 0) extra[team][c[s]] = 0.0f;
            __syncwarp();
        }
    }
}

template <class... KArgs> unsigned resident_blocks(void (*kernel)(KArgs...))
{
    int n = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, ROUTE_BLOCK, 0) != cudaSuccess) cudaGetLastError();
    return n > 0 ? (unsigned)n : 1u;
}

uint32_t route_teams(uint32_t experts) { return experts <= 16 ? 64 : experts <= 128 ? 32 : experts <= 256 ? 16 : 8; }      // at least
// Blocks at most (launch_clusters may find that fewer fit): a rule on the sizes and the device alone, so that the order of the
// additions is theirs too.
unsigned route_blocks(const nups_store* s, uint64_t n, uint32_t experts)
{
    const unsigned blocks = grid_for(n, route_teams(experts), (unsigned)s->sm_count * (experts <= 64 ? 4 : experts <= 512 ? 3 : 2));
    return blocks == 1 ? 1 : blocks < ROUTE_CLUSTER ? ROUTE_CLUSTER : blocks / ROUTE_CLUSTER * ROUTE_CLUSTER;       // whole clusters
}

// Do rows of logits allow runs of VEC?
bool route_wide(const void* p, uint64_t stride, uint32_t experts, uint64_t n, int bytes, int vec)
{
    return experts % vec == 0 && ((uintptr_t)p & (bytes * vec - 1)) == 0 && (n <= 1 || stride % vec == 0);
}

// Blocks in clusters of ROUTE_CLUSTER, as many as fit on the device at once; a single block by itself.
cudaError_t launch_clusters(void (*kernel)(RouteArgs), std::atomic<uint32_t>& fit, unsigned& blocks, cudaStream_t st, const RouteArgs& a)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(ROUTE_BLOCK);
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = ROUTE_CLUSTER;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = blocks == 1 ? 1 : 2;
    if (blocks > ROUTE_CLUSTER) {                           // asked for once per kernel
        uint32_t most = fit.load(std::memory_order_relaxed);
        if (!most) {
            int n = 0;
            const cudaError_t e = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
            if (e != cudaSuccess) return e;
            most = n > 0 ? (uint32_t)n : 1u;
            fit.store(most, std::memory_order_relaxed);
        }
        if (blocks > most * ROUTE_CLUSTER) blocks = most * ROUTE_CLUSTER;
        cfg.gridDim = dim3(blocks);
    }
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <class X>
nups_status launch_route(nups_store* s, const RouteArgs& a, cudaStream_t st)
{
    unsigned blocks = route_blocks(s, a.n, a.experts);
    constexpr int V = 16 / sizeof(X);
    const bool wide = route_wide(a.logits, a.stride, a.experts, a.n, sizeof(X), a.experts <= 16 ? 4 : V);
    // KEPT: as many as a lane is at all likely to give (a lane that gives more looks through its logits again)
#define NUPS_ROUTE_KEPT(TPR_, EPT_, V_, KEPT_)                                                                        \
    {                                                                                                                 \
        static std::atomic<uint32_t> fit[2];                                                                          \
        if (wide) CK(launch_clusters(route_kernel<X, V_, TPR_, EPT_, KEPT_>, fit[0], blocks, st, a));                 \
        else CK(launch_clusters(route_kernel<X, 1, TPR_, EPT_, KEPT_>, fit[1], blocks, st, a));                       \
    }
#define NUPS_ROUTE(TPR_, EPT_, V_)                                                                                    \
    {                                                                                                                 \
        if (a.top == 1) NUPS_ROUTE_KEPT(TPR_, EPT_, V_, 1)                                                            \
        else if (a.top <= 2 || sizeof(X) == 4 || EPT_ < 8) NUPS_ROUTE_KEPT(TPR_, EPT_, V_, 2)                         \
        else if constexpr (sizeof(X) == 2 && EPT_ >= 8) NUPS_ROUTE_KEPT(TPR_, EPT_, V_, 4)                            \
    }
    if (a.experts <= 16) NUPS_ROUTE(4, 4, 4)
    else if (a.experts <= 64) NUPS_ROUTE(8, 8, V)
    else if (a.experts <= 128) NUPS_ROUTE(8, 16, V)
    else if (a.experts <= 256) NUPS_ROUTE((sizeof(X) == 2 ? 8 : 16), (sizeof(X) == 2 ? 32 : 16), V)
    else if (a.experts <= 512) NUPS_ROUTE((sizeof(X) == 2 ? 16 : 32), (sizeof(X) == 2 ? 32 : 16), V)
    else NUPS_ROUTE(32, 32, V)
#undef NUPS_ROUTE
#undef NUPS_ROUTE_KEPT
    LAUNCH_CHECK(s);
    if (blocks == 1) return NUPS_OK;
    uint32_t width = 32;
    while (width * JOIN_CLUSTER < a.experts) width *= 2;
    nups_launch_dependent(route_join_kernel, JOIN_CLUSTER, JOIN_BLOCK, 0, st, a, blocks / ROUTE_CLUSTER, width);
    LAUNCH_CHECK(s);
    return NUPS_OK;
}

template <class X>
nups_status launch_route_grad(nups_store* s, const RouteGradArgs& a, cudaStream_t st)
{
    constexpr int V = 16 / sizeof(X);
    const int v = a.experts <= 16 ? 4 : V;
    const bool wide = route_wide(a.logits, a.stride, a.experts, a.n, sizeof(X), v) && route_wide(a.dlogits, a.dstride, a.experts, a.n, sizeof(X), v);
#define NUPS_ROUTE(TPR_, EPT_, V_)                                                                                                     \
    {                                                                                                                                  \
        static const unsigned resident = resident_blocks(route_grad_kernel<X, V_, TPR_, EPT_>);                                        \
        const unsigned blocks = grid_for(a.n, ROUTE_BLOCK / TPR_, (unsigned)s->sm_count * resident);                                   \
        if (wide) nups_launch_dependent(route_grad_kernel<X, V_, TPR_, EPT_>, blocks, ROUTE_BLOCK, 0, st, a);                          \
        else nups_launch_dependent(route_grad_kernel<X, 1, TPR_, EPT_>, blocks, ROUTE_BLOCK, 0, st, a);                                \
    }
    if (a.experts <= 16) NUPS_ROUTE(4, 4, 4)
    else if (a.experts <= 64) NUPS_ROUTE(8, 8, V)
    else if (a.experts <= 128) NUPS_ROUTE(8, 16, V)
    else if (a.experts <= 256) NUPS_ROUTE((sizeof(X) == 2 ? 8 : 16), (sizeof(X) == 2 ? 32 : 16), V)
    else if (a.experts <= 512) NUPS_ROUTE((sizeof(X) == 2 ? 16 : 32), (sizeof(X) == 2 ? 32 : 16), V)
    else NUPS_ROUTE(32, 32, V)
#undef NUPS_ROUTE
    LAUNCH_CHECK(s);
    return NUPS_OK;
}

bool route_sizes(int type, uint64_t stride, uint64_t n, uint32_t experts, uint32_t top, float balance, float z)
{
    return (type == NUPS_F32 || type == NUPS_F16 || type == NUPS_BF16) && experts >= 1 && experts <= NUPS_ROUTE_MAX_EXPERTS && top >= 1 && top <= experts &&
           top <= NUPS_ROUTE_MAX_TOP && n < (1ull << 32) && stride < (1ull << 32) && (n <= 1 || stride >= experts) && isfinite(balance) && isfinite(z);
}

}  // namespace

extern "C" nups_status nups_route_scratch(nups_store* s, uint64_t n, uint32_t experts, uint64_t* h_bytes_out)
{
    if (!s || !h_bytes_out || experts < 1 || experts > NUPS_ROUTE_MAX_EXPERTS || n >= (1ull << 32)) return NUPS_EINVAL;
    const uint64_t groups = route_blocks(s, n, experts) / ROUTE_CLUSTER;
    *h_bytes_out = groups * (experts + 1) * 8;           // one block finishes by itself
    return NUPS_OK;
}

extern "C" nups_status nups_route(nups_store* s, const void* d_logits, int type, uint64_t stride, uint64_t n, uint32_t experts, uint32_t top,
                                  const uint8_t* d_active, int renormalize, float balance, float z, int32_t* d_choice, float* d_weight,
                                  float* d_lse, uint64_t* d_counts, uint64_t* d_tokens, float* d_prob, float* d_loss, void* d_scratch,
                                  uint64_t scratch_bytes, void* stream)
{
    if (!s || !route_sizes(type, stride, n, experts, top, balance, z) || !d_counts || !d_tokens) return NUPS_EINVAL;
    if (n && (!d_logits || !d_choice || !d_weight)) return NUPS_EINVAL;
    if (!suits(type_bytes(type), d_logits) || !suits(4, d_choice, d_weight, d_lse, d_prob, d_loss) || !suits(8, d_counts, d_tokens)) return NUPS_EINVAL;
    uint64_t bytes = 0;
    nups_route_scratch(s, n, experts, &bytes);
    if (bytes && (!d_scratch || scratch_bytes < bytes || ((uintptr_t)d_scratch & 255))) return NUPS_EINVAL;
    nups_status rc = on_own_device(s);
    if (rc != NUPS_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    if (n == 0) {
        CK(cudaMemsetAsync(d_counts, 0, experts * sizeof(uint64_t), st));
        CK(cudaMemsetAsync(d_tokens, 0, sizeof(uint64_t), st));
        if (d_prob) CK(cudaMemsetAsync(d_prob, 0, experts * sizeof(float), st));
        if (d_loss) CK(cudaMemsetAsync(d_loss, 0, 3 * sizeof(float), st));
        return NUPS_OK;
    }
    const uint64_t cells = (uint64_t)(route_blocks(s, n, experts) / ROUTE_CLUSTER) * (experts + 1);
    RouteArgs a = {d_logits, stride, n, experts, top, d_active, renormalize != 0, d_prob || d_loss, balance, z, d_choice, d_weight, d_lse, d_counts, d_tokens,
                   d_prob, d_loss, (float*)d_scratch, (uint32_t*)d_scratch + cells};
    return type == NUPS_F32 ? launch_route<float>(s, a, st) : type == NUPS_F16 ? launch_route<__half>(s, a, st) : launch_route<__nv_bfloat16>(s, a, st);
}

extern "C" nups_status nups_route_grad(nups_store* s, const void* d_logits, int type, uint64_t stride, uint64_t n, uint32_t experts, uint32_t top,
                                       const uint8_t* d_active, int renormalize, float balance, float z, const int32_t* d_choice,
                                       const float* d_weight, const float* d_lse, const uint64_t* d_counts, const uint64_t* d_tokens, const float* d_dloss,
                                       const float* d_dweight, void* d_dlogits, uint64_t dlogits_stride, void* stream)
{
    if (!s || !route_sizes(type, stride, n, experts, top, balance, z) || !route_sizes(type, dlogits_stride, n, experts, top, 0, 0)) return NUPS_EINVAL;
    if (n && (!d_logits || !d_lse || !d_counts || !d_tokens || !d_dlogits || (d_dweight && (!d_choice || !d_weight)))) return NUPS_EINVAL;
    if (!suits(type_bytes(type), d_logits, d_dlogits) || !suits(4, d_choice, d_weight, d_lse, d_dloss, d_dweight) || !suits(8, d_counts, d_tokens)) return NUPS_EINVAL;
    nups_status rc = on_own_device(s);
    if (rc != NUPS_OK || n == 0) return rc;
    RouteGradArgs a = {d_logits, stride, n, experts, top, d_active, renormalize != 0, balance, z, d_choice, d_weight, d_lse, d_counts, d_tokens, d_dloss, d_dweight,
                       d_dlogits, dlogits_stride};
    cudaStream_t st = (cudaStream_t)stream;
    return type == NUPS_F32 ? launch_route_grad<float>(s, a, st)
                            : type == NUPS_F16 ? launch_route_grad<__half>(s, a, st) : launch_route_grad<__nv_bfloat16>(s, a, st);
}
