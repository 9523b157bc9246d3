// The balance loss of a router over batches of tokens (one batch a rank),
// the counts that go with it, and its gradient.
//
// A batch has T tokens that chose at least one of the E experts, k choices
// each.  With p = softmax(logits) of a token, n_i the choices of expert i and
// s_d the tokens that chose an expert of rank d (E / D experts each):
//
//   f_i = n_i E / (k T)    P_i = mean of p_i over the T tokens
//   w_i = a f_i + b (mean of f over the experts of i's rank) + c s_d D / (M T)
//   loss = sum of w_i P_i            (sums over a rank's P are in the w)
//
// f and s are counts and carry no gradient; with the loss's gradient g,
//
//   dlogit_j = g / T p_j (w_j - sum of w_i p_i) .
//
// As p sums to one, a constant taken off w changes nothing there: what the
// backward pass reads is (w_i - mean of w) / T, made in 64 bits, since a
// balanced router's w are nearly the same and the gradient lives on their
// differences.  A token without a choice in [0, E) is padding: it is in no
// sum and its gradient is zero, whatever its logits hold.  A token whose
// logits are all -inf has p = 0.
//
// L lanes hold a token's logits, 4 (or up to 16) each; the sums over tokens
// stay in registers and are joined once a workgroup; choices are counted in
// LDS, in integers, whose order does not matter.  The partial sums of the
// workgroups, a number that goes by the sizes alone, are added in order by
// one workgroup a batch.
//
// Bound by memory at many tokens (logits and choices read once, gradients
// written), by the launches and the last sum's latency at few.
#include <type_traits>

#include "lanes.h"
#include "shard_ops.h"

namespace hoccl {
namespace {

constexpr int kWaves = kOpThreads / 64;
constexpr float kLog2e = 1.4426950408889634f;

// Lanes of a token and vectors of 4 logits a lane.
constexpr int vectors_of(int E) { return E <= 256 ? 1 : E <= 512 ? 2 : 4; }
int lanes_of(int E) {
    int l = 1;
    while (l < 64 && l * 4 < E) l *= 2;
    return l;
}

__device__ __forceinline__ int choice(const BalanceArgs &a, const BalanceSeg &s, uint64_t i) {
    // What does not fit in 31 bits is no expert either.
    if (a.index64) {
        const int64_t v = ((const int64_t *)s.experts)[i];
        return v >= 0 && v < a.E ? (int)v : -1;
    }
    const int32_t v = ((const int32_t *)s.experts)[i];
    return v >= 0 && v < a.E ? v : -1;
}

// p = softmax of the L lanes' logits; behind E it is 0.
template <int L, int NV>
__device__ __forceinline__ void softmax(float (&x)[NV][4], int lane, int E) {
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if ((j * L + lane) * 4 + i >= E) x[j][i] = -INFINITY;
            top = fmaxf(top, x[j][i]);
        }
    top = join_lanes<L, LaneMax>(top);
    // All -inf: -inf - 0 below leaves p = 0.
    const float base = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[j][i] = __builtin_amdgcn_exp2f((x[j][i] - base) * kLog2e);
            sum += x[j][i];
        }
    sum = join_lanes<L, LaneSum>(sum);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[j][i] *= inv;
}

// Loss, weights and counts of batch `seg` from its blocks' sums.
__device__ void finish(const BalanceArgs &a, int seg, double *wsum, int *nsum, double (*red)[2]) {
    const int E = a.E, D = a.D, per = E / D, stride = E + D + 1;
    const uint32_t b0 = a.first[seg], b1 = a.first[seg + 1];
    const int t = threadIdx.x, nt = blockDim.x;
    // nsum: choices of E experts, tokens of D ranks, tokens.
    for (int e = t; e < stride; e += nt) {
        int n = 0;
        for (uint32_t b = b0; b < b1; ++b) n += a.partial_n[(uint64_t)b * stride + e];
        nsum[e] = n;
        if (e < E) a.expert_tokens[(uint64_t)seg * E + e] = n;
        else if (e < E + D) a.rank_tokens[(uint64_t)seg * D + e - E] = n;
    }
    __syncthreads();
    const double T = nsum[E + D] > 0 ? (double)nsum[E + D] : 1.0;
    double loss = 0.0, all = 0.0;
    for (int e = t; e < E; e += nt) {
        const int d = e / per;
        int group = 0;
        for (int i = d * per; i < (d + 1) * per; ++i) group += nsum[i];
        const double f = (double)E / ((double)a.k * T);
        const double w = a.expert_weight * f * nsum[e] + a.rank_weight * f * group / per +
                         a.traffic_weight * (double)D * nsum[E + d] / ((double)a.max_ranks * T);
        double p = 0.0;
        for (uint32_t b = b0; b < b1; ++b) p += (double)a.partial_p[(uint64_t)b * E + e];
        loss += w * p / T;
        all += w;
        wsum[e] = w;
    }
    // The threads' sums in a fixed order.
    for (int o = 32; o > 0; o /= 2) {
        loss += __shfl_xor(loss, o);
        all += __shfl_xor(all, o);
    }
    if (t % 64 == 0) red[t / 64][0] = loss, red[t / 64][1] = all;
    __syncthreads();
    loss = 0.0, all = 0.0;
    for (int i = 0; i < nt / 64; ++i) loss += red[i][0], all += red[i][1];
    for (int e = t; e < E; e += nt)
        a.coef[(uint64_t)seg * E + e] = nsum[E + D] > 0 ? (float)((wsum[e] - all / E) / T) : 0.0f;
    if (t == 0) a.loss[seg] = (float)loss;
    __syncthreads();
}

template <class T, int L, int NV>
__global__ void __launch_bounds__(kOpThreads) balance_kernel(BalanceArgs) {
    const BalanceArgs &a = kernel_args<BalanceArgs>();
    constexpr int ROWS = kOpThreads / L;   // tokens of a workgroup's pass
    constexpr int OWN = L == 64 ? 1 : 4;   // ranks a lane counts: D <= 4 L, and D <= 64
    __shared__ float sum_p[kWaves][L * NV * 4];
    __shared__ int sum_n[L * NV * 4];
    __shared__ int sum_sent[64];
    __shared__ int sum_live;
    const int E = a.E, D = a.D, k = a.k, per = E / D, stride = E + D + 1;
    const int lane = threadIdx.x % L, slot = threadIdx.x / L;
    for (uint32_t block = blockIdx.x; block < a.first[a.nseg]; block += gridDim.x) {
        int seg = 0;
        while (a.first[seg + 1] <= block) ++seg;
        const BalanceSeg &s = a.seg[seg];
        const uint32_t nb = a.first[seg + 1] - a.first[seg], lb = block - a.first[seg];
        for (int e = threadIdx.x; e < E; e += kOpThreads) sum_n[e] = 0;
        if (threadIdx.x < 64) sum_sent[threadIdx.x] = 0;
        if (threadIdx.x == 0) sum_live = 0;
        __syncthreads();
        float acc[NV][4] = {};
        int sent[OWN] = {}, live = 0;
        for (uint64_t row0 = (uint64_t)lb * ROWS; row0 < s.tokens; row0 += (uint64_t)nb * ROWS) {
            // Every lane stays for the exchanges; a row behind the last
            // reads nothing and is padding.
            const uint64_t row = row0 + slot;
            const bool in = row < s.tokens;
            float x[NV][4];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int e = (j * L + lane) * 4;
                load_some<T>((const char *)s.logits + row * E * T::size, e, in ? E : 0, x[j]);
            }
            uint32_t lo = 0, hi = 0;  // the ranks that the token goes to
            bool any = false;
            for (int c = lane; c < k; c += L) {
                const int e = in ? choice(a, s, row * k + c) : -1;
                if (e < 0) continue;
                any = true;
                const int d = e / per;
                if (d < 32) lo |= 1u << d;
                else hi |= 1u << (d - 32);
                atomicAdd(&sum_n[e], 1);
            }
            const bool valid = join_lanes<L, LaneOr>((uint32_t)any) != 0;
            lo = join_lanes<L, LaneOr>(lo);
            if (D > 32) hi = join_lanes<L, LaneOr>(hi);
            if (lane == 0) live += valid;
#pragma unroll
            for (int i = 0; i < OWN; ++i) {
                const int d = i * L + lane;
                sent[i] += d < 32 ? (lo >> d) & 1u : d < 64 ? (hi >> (d - 32)) & 1u : 0;
            }
            softmax<L, NV>(x, lane, E);
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j][i] += valid ? x[j][i] : 0.0f;
        }
        // The wave's groups, then the waves in order.
#pragma unroll
        for (int o = L; o < 64; o *= 2)
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j][i] += __shfl_xor(acc[j][i], o);
        if (threadIdx.x % 64 < L)
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum_p[threadIdx.x / 64][(j * L + lane) * 4 + i] = acc[j][i];
#pragma unroll
        for (int i = 0; i < OWN; ++i)
            if (i * L + lane < D && sent[i]) atomicAdd(&sum_sent[i * L + lane], sent[i]);
        if (live) atomicAdd(&sum_live, live);
        __syncthreads();
        int32_t *pn = a.partial_n + (uint64_t)block * stride;
        for (int e = threadIdx.x; e < E; e += kOpThreads) {
            float p = 0.0f;
            for (int w = 0; w < kWaves; ++w) p += sum_p[w][e];
            a.partial_p[(uint64_t)block * E + e] = p;
            pn[e] = sum_n[e];
        }
        if ((int)threadIdx.x < D) pn[E + threadIdx.x] = sum_sent[threadIdx.x];
        if (threadIdx.x == 0) pn[E + D] = sum_live;
        __syncthreads();
    }
}

constexpr int kFinishThreads = 1024;
__global__ void __launch_bounds__(kFinishThreads) balance_finish_kernel(BalanceArgs) {
    const BalanceArgs &a = kernel_args<BalanceArgs>();
    __shared__ double wsum[kMaxExperts];
    __shared__ int nsum[kMaxExperts + 64 + 1];
    __shared__ double red[kFinishThreads / 64][2];
    for (int seg = blockIdx.x; seg < a.nseg; seg += gridDim.x) finish(a, seg, wsum, nsum, red);
}

template <class T, int L, int NV>
__global__ void __launch_bounds__(kOpThreads) balance_backward_kernel(BalanceArgs) {
    const BalanceArgs &a = kernel_args<BalanceArgs>();
    constexpr int ROWS = kOpThreads / L;
    const int E = a.E, k = a.k;
    const int lane = threadIdx.x % L, slot = threadIdx.x / L;
    for (uint32_t block = blockIdx.x; block < a.first[a.nseg]; block += gridDim.x) {
        int seg = 0;
        while (a.first[seg + 1] <= block) ++seg;
        const BalanceSeg &s = a.seg[seg];
        const uint32_t nb = a.first[seg + 1] - a.first[seg], lb = block - a.first[seg];
        float w[NV][4];
#pragma unroll
        for (int j = 0; j < NV; ++j) load_some<EF32>(a.coef + (uint64_t)seg * E, (j * L + lane) * 4, E, w[j]);
        const float g = a.grad ? a.grad[seg] : 1.0f;
        for (uint64_t row0 = (uint64_t)lb * ROWS; row0 < s.tokens; row0 += (uint64_t)nb * ROWS) {
            const uint64_t row = row0 + slot;
            const bool in = row < s.tokens;
            float x[NV][4];
#pragma unroll
            for (int j = 0; j < NV; ++j)
                load_some<T>((const char *)s.logits + row * E * T::size, (j * L + lane) * 4, in ? E : 0, x[j]);
            bool any = false;
            for (int c = lane; c < k; c += L) any |= in && choice(a, s, row * k + c) >= 0;
            const bool valid = join_lanes<L, LaneOr>((uint32_t)any) != 0;
            softmax<L, NV>(x, lane, E);
            float dot = 0.0f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) dot += x[j][i] * w[j][i];
            dot = join_lanes<L, LaneSum>(dot);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float d[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) d[i] = valid ? g * x[j][i] * (w[j][i] - dot) : 0.0f;
                store_some<T>((char *)s.dlogits + row * E * T::size, (j * L + lane) * 4, in ? E : 0, d);
            }
        }
    }
}

// f(T, L, NV) of the logits' type and the number of experts.
template <class F>
const void *with_lanes(hoccl_dtype_t dt, int E, F &&f) {
    auto typed = [&](auto l, auto nv) { return dt == HOCCL_BF16 ? f(EBF16(), l, nv) : f(EF32(), l, nv); };
#define HOCCL_LANES(l, n) return typed(std::integral_constant<int, l>(), std::integral_constant<int, n>())
    switch (vectors_of(E)) {
    case 2: HOCCL_LANES(64, 2);
    case 4: HOCCL_LANES(64, 4);
    }
    switch (lanes_of(E)) {
    case 1: HOCCL_LANES(1, 1);
    case 2: HOCCL_LANES(2, 1);
    case 4: HOCCL_LANES(4, 1);
    case 8: HOCCL_LANES(8, 1);
    case 16: HOCCL_LANES(16, 1);
    case 32: HOCCL_LANES(32, 1);
    }
    HOCCL_LANES(64, 1);
#undef HOCCL_LANES
}

// Workgroups of one batch, each with at least `passes` passes over its rows.
uint32_t blocks_of(size_t tokens, int E, size_t passes, size_t most) {
    const size_t rows = (size_t)(kOpThreads / lanes_of(E)) * passes, n = (tokens + rows - 1) / rows;
    return (uint32_t)(n < 1 ? 1 : n < most ? n : most);
}

}  // namespace

uint32_t balance_blocks(size_t tokens, int E, int batches) {
    return blocks_of(tokens, E, 4, batches < 8 ? 512 / batches : 64);
}

hipError_t launch_balance(const BalanceArgs &a, hoccl_dtype_t dt, int wg, hipStream_t s) {
    const void *k = with_lanes(dt, a.E, [](auto t, auto l, auto n) {
        return (const void *)balance_kernel<decltype(t), decltype(l)::value, decltype(n)::value>;
    });
    void *args[] = {(void *)&a};
    return hipLaunchKernel(k, dim3((unsigned)wg), dim3(kOpThreads), args, 0, s);
}

hipError_t launch_balance_finish(const BalanceArgs &a, int wg, hipStream_t s) {
    void *args[] = {(void *)&a};
    return hipLaunchKernel((const void *)balance_finish_kernel, dim3((unsigned)wg), dim3(kFinishThreads), args, 0, s);
}

uint32_t balance_backward_blocks(size_t tokens, int E) { return blocks_of(tokens, E, 1, 4096); }

hipError_t launch_balance_backward(const BalanceArgs &a, hoccl_dtype_t dt, int wg, hipStream_t s) {
    const void *k = with_lanes(dt, a.E, [](auto t, auto l, auto n) {
        return (const void *)balance_backward_kernel<decltype(t), decltype(l)::value, decltype(n)::value>;
    });
    void *args[] = {(void *)&a};
    return hipLaunchKernel(k, dim3((unsigned)wg), dim3(kOpThreads), args, 0, s);
}

}  // namespace hoccl
