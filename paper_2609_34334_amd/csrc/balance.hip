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
// L lanes hold a token's logits, 8 each (16 of more than 512 experts), in
// vectors of 16 bytes; two tokens of every lane are in flight.  The sums over
// tokens stay in registers and are joined once a workgroup; choices are
// counted in LDS, in integers, whose order does not matter.  The partial sums
// of the workgroups, a number that goes by the sizes alone, are added in order
// by one workgroup a batch.
//
// Bound by memory at many tokens (logits and choices read once, gradients
// written), by the launches and the last sum's latency at few.
#include <type_traits>

#include "lanes.h"
#include "shard_ops.h"

namespace hoccl {
namespace {

constexpr int kThreads = 512;  // of the forward pass's first kernel
constexpr int kWaves = kThreads / 64;
constexpr int kAhead = 2;      // tokens of a lane in flight
constexpr float kLog2e = 1.4426950408889634f;

int lanes_of(int E) {
    int l = 1;
    while (l < 64 && l * 8 < E) l *= 2;
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

// A lane's logits of one token: NV vectors of VE, L lanes apart.
template <class T, int L, int N>
struct Logits {
    static constexpr int VE = 16 / T::size, NV = N / VE;
    float v[NV][VE];
    static __device__ __forceinline__ int at(int j, int lane) { return (j * L + lane) * VE; }
    // `E`: 0 reads nothing.
    __device__ __forceinline__ void load(const void *p, int lane, int E) {
#pragma unroll
        for (int j = 0; j < NV; ++j) load_some<T>(p, at(j, lane), E, v[j]);
    }
    __device__ __forceinline__ void store(void *p, int lane, int E) const {
#pragma unroll
        for (int j = 0; j < NV; ++j) store_some<T>(p, at(j, lane), E, v[j]);
    }
    // To exp(x - max) over the L lanes; returns what makes them p: the
    // reciprocal (1 ulp) of their sum.  Behind E there are zeros.
    __device__ __forceinline__ float softmax(int lane, int E) {
        float top = -INFINITY, sum = 0.0f;
        if (E < L * N)
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VE; ++i)
                    if (at(j, lane) + i >= E) v[j][i] = -INFINITY;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VE; ++i) top = fmaxf(top, v[j][i]);
        top = join_lanes<L, LaneMax>(top);
        // All -inf: -inf - 0 leaves p = 0.
        const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                v[j][i] = __builtin_amdgcn_exp2f((v[j][i] - base) * kLog2e);
                sum += v[j][i];
            }
        sum = join_lanes<L, LaneSum>(sum);
        return sum == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(sum);
    }
};

// The batch of a block, and its place among the batch's blocks.
__device__ __forceinline__ int batch_of(const BalanceArgs &a, uint32_t block, uint32_t &lb, uint32_t &nb) {
    int seg = 0;
    while (a.first[seg + 1] <= block) ++seg;
    nb = a.first[seg + 1] - a.first[seg], lb = block - a.first[seg];
    return seg;
}

template <class T, int L, int N>
__global__ void __launch_bounds__(kThreads) balance_kernel(BalanceArgs) {
    const BalanceArgs &a = kernel_args<BalanceArgs>();
    using X = Logits<T, L, N>;
    constexpr int ROWS = kThreads / L;     // tokens of a workgroup's pass, kAhead times
    constexpr int OWN = L < 8 ? 8 : 64 / L;  // ranks a lane counts: no more than its experts, nor 64 in all
    __shared__ float sum_p[kWaves][L * N];
    __shared__ int sum_n[L * N];
    __shared__ int sum_sent[64];
    __shared__ int sum_live;
    const int E = a.E, D = a.D, k = a.k, stride = 2 * E + D + 1;
    const int lane = threadIdx.x % L, slot = threadIdx.x / L;
    for (uint32_t block = blockIdx.x; block < a.first[a.nseg]; block += gridDim.x) {
        uint32_t lb, nb;
        const BalanceSeg &s = a.seg[batch_of(a, block, lb, nb)];
        for (int e = threadIdx.x; e < E; e += kThreads) sum_n[e] = 0;
        if (threadIdx.x < 64) sum_sent[threadIdx.x] = 0;
        if (threadIdx.x == 0) sum_live = 0;
        __syncthreads();
        float acc[X::NV][X::VE] = {};
        int sent[OWN] = {}, live = 0;
        for (uint64_t row0 = (uint64_t)lb * ROWS * kAhead; row0 < s.tokens; row0 += (uint64_t)nb * ROWS * kAhead) {
            // Every lane stays for the exchanges; a row behind the last
            // reads nothing and is padding.
            X x[kAhead];
            int first[kAhead];  // the lane's first choice
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint64_t row = row0 + u * ROWS + slot;
                const bool in = row < s.tokens;
                x[u].load((const char *)s.logits + row * E * T::size, lane, in ? E : 0);
                first[u] = in && lane < k ? choice(a, s, row * k + lane) : -1;
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint64_t row = row0 + u * ROWS + slot;
                const bool in = row < s.tokens;
                uint32_t lo = 0, hi = 0;  // the ranks that the token goes to
                bool any = false;
                auto choose = [&](int e) {
                    if (e < 0) return;
                    any = true;
                    const uint32_t d = ((uint32_t)e * a.rank_mul) >> 21;
                    if (d < 32) lo |= 1u << d;
                    else hi |= 1u << (d - 32);
                    atomicAdd(&sum_n[e], 1);
                };
                choose(first[u]);
                for (int c = lane + L; c < k; c += L)
                    if (in) choose(choice(a, s, row * k + c));
                const bool valid = join_lanes<L, LaneOr>((uint32_t)any) != 0;
                lo = join_lanes<L, LaneOr>(lo);
                if (D > 32) hi = join_lanes<L, LaneOr>(hi);
                if (lane == 0) live += valid;
#pragma unroll
                for (int i = 0; i < OWN; ++i) {
                    const int d = i * L + lane;
                    sent[i] += ((d < 32 ? lo : hi) >> (d & 31)) & 1u;
                }
                const float inv = x[u].softmax(lane, E);
#pragma unroll
                for (int j = 0; j < X::NV; ++j)
#pragma unroll
                    for (int i = 0; i < X::VE; ++i) acc[j][i] += valid ? x[u].v[j][i] * inv : 0.0f;
            }
        }
        // The wave's groups, then the waves in order.
#pragma unroll
        for (int o = L; o < 64; o *= 2)
#pragma unroll
            for (int j = 0; j < X::NV; ++j)
#pragma unroll
                for (int i = 0; i < X::VE; ++i) acc[j][i] += __shfl_xor(acc[j][i], o);
        if (threadIdx.x % 64 < L)
#pragma unroll
            for (int j = 0; j < X::NV; ++j)
#pragma unroll
                for (int i = 0; i < X::VE; ++i) sum_p[threadIdx.x / 64][X::at(j, lane) + i] = acc[j][i];
#pragma unroll
        for (int i = 0; i < OWN; ++i)
            if (sent[i]) atomicAdd(&sum_sent[i * L + lane], sent[i]);
        if (live) atomicAdd(&sum_live, live);
        __syncthreads();
        int32_t *out = a.partial + (uint64_t)block * stride;
        for (int e = threadIdx.x; e < E; e += kThreads) {
            float p = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) p += sum_p[w][e];
            out[e] = __float_as_int(p);
            out[E + e] = sum_n[e];
        }
        if ((int)threadIdx.x < D) out[2 * E + threadIdx.x] = sum_sent[threadIdx.x];
        if (threadIdx.x == 0) out[2 * E + D] = sum_live;
        __syncthreads();
    }
}

// Loss, weights and counts of a batch from its blocks' sums.  The sums of p,
// the counts of choices, of tokens a rank and of tokens are columns of one
// table with a row a block; all are added in 64 bits, where the counts are
// exact.  Lots of rows are added side by side, eight rows of each in flight,
// then the lots in order: one row after another, 64 blocks took 35 us, all
// latency.
constexpr int kFinishThreads = 1024;
constexpr int kColumns = 2 * kMaxExperts + 64 + 1;
__global__ void __launch_bounds__(kFinishThreads) balance_finish_kernel(BalanceArgs) {
    const BalanceArgs &a = kernel_args<BalanceArgs>();
    __shared__ double lot[kFinishThreads];
    __shared__ double tot[kColumns];
    __shared__ double rank_choices[64];
    __shared__ double red[kFinishThreads / 64][2];
    const int E = a.E, D = a.D, per = E / D, cols = 2 * E + D + 1, t = threadIdx.x;
    const int wide = (cols + 63) / 64 * 64;
    const int lots = wide < kFinishThreads ? kFinishThreads / wide : 1;
    for (int seg = blockIdx.x; seg < a.nseg; seg += gridDim.x) {
        const uint32_t nb = a.first[seg + 1] - a.first[seg];
        const int32_t *rows = a.partial + (uint64_t)a.first[seg] * cols;
        const int g = lots > 1 ? t / wide : 0;
        for (int c = lots > 1 ? t % wide : t; c < cols; c += lots > 1 ? wide : kFinishThreads) {
            if (g >= lots) break;
            double sum = 0.0;
            for (uint32_t b0 = g; b0 < nb; b0 += 8 * lots) {
                int32_t v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t b = b0 + i * lots;
                    v[i] = b < nb ? rows[(uint64_t)b * cols + c] : 0;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += c < E ? (double)__int_as_float(v[i]) : (double)v[i];
            }
            if (lots > 1) lot[t] = sum;
            else tot[c] = sum;
        }
        __syncthreads();
        if (lots > 1 && t < cols) {
            double sum = lot[t];
            for (int i = 1; i < lots; ++i) sum += lot[i * wide + t];
            tot[t] = sum;
        }
        __syncthreads();
        for (int e = t; e < E; e += kFinishThreads) a.expert_tokens[(uint64_t)seg * E + e] = (int32_t)tot[E + e];
        if (t < D) a.rank_tokens[(uint64_t)seg * D + t] = (int32_t)tot[2 * E + t];
        for (int d = t / 64; d < D; d += kFinishThreads / 64) {  // a wave a rank
            double n = 0.0;
            for (int e = d * per + t % 64; e < (d + 1) * per; e += 64) n += tot[E + e];
#pragma unroll
            for (int o = 32; o > 0; o /= 2) n += __shfl_xor(n, o);
            if (t % 64 == 0) rank_choices[d] = n;
        }
        __syncthreads();
        const double live = tot[2 * E + D], T = live > 0.0 ? live : 1.0;
        double loss = 0.0, all = 0.0, w = 0.0;
        if (t < E) {
            const int d = t / per;
            const double f = (double)E / ((double)a.k * T);
            w = a.expert_weight * f * tot[E + t] + a.rank_weight * f * rank_choices[d] / per +
                a.traffic_weight * (double)D * tot[2 * E + d] / ((double)a.max_ranks * T);
            loss = w * tot[t] / T;
            all = w;
        }
#pragma unroll
        for (int o = 32; o > 0; o /= 2) {
            loss += __shfl_xor(loss, o);
            all += __shfl_xor(all, o);
        }
        if (t % 64 == 0) red[t / 64][0] = loss, red[t / 64][1] = all;
        __syncthreads();
        loss = 0.0, all = 0.0;
        for (int i = 0; i < (E + 63) / 64; ++i) loss += red[i][0], all += red[i][1];
        if (t < E) a.coef[(uint64_t)seg * E + t] = live > 0.0 ? (float)((w - all / E) / T) : 0.0f;
        if (t == 0) a.loss[seg] = (float)loss;
        __syncthreads();
    }
}
static_assert(kMaxExperts <= kFinishThreads, "a thread an expert");

template <class T, int L, int N>
__global__ void __launch_bounds__(kOpThreads) balance_backward_kernel(BalanceArgs) {
    const BalanceArgs &a = kernel_args<BalanceArgs>();
    using X = Logits<T, L, N>;
    constexpr int ROWS = kOpThreads / L;
    const int E = a.E, k = a.k;
    const int lane = threadIdx.x % L, slot = threadIdx.x / L;
    for (uint32_t block = blockIdx.x; block < a.first[a.nseg]; block += gridDim.x) {
        uint32_t lb, nb;
        const int seg = batch_of(a, block, lb, nb);
        const BalanceSeg &s = a.seg[seg];
        float w[X::NV][X::VE];
#pragma unroll
        for (int j = 0; j < X::NV; ++j) load_some<EF32>(a.coef + (uint64_t)seg * E, X::at(j, lane), E, w[j]);
        const float g = a.grad ? a.grad[seg] : 1.0f;
        for (uint64_t row0 = (uint64_t)lb * ROWS * kAhead; row0 < s.tokens; row0 += (uint64_t)nb * ROWS * kAhead) {
            X x[kAhead];
            bool any[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint64_t row = row0 + u * ROWS + slot;
                const bool in = row < s.tokens;
                x[u].load((const char *)s.logits + row * E * T::size, lane, in ? E : 0);
                any[u] = in && lane < k && choice(a, s, row * k + lane) >= 0;
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint64_t row = row0 + u * ROWS + slot;
                const bool in = row < s.tokens;
                for (int c = lane + L; c < k; c += L) any[u] |= in && choice(a, s, row * k + c) >= 0;
                const bool valid = join_lanes<L, LaneOr>((uint32_t)any[u]) != 0;
                const float inv = x[u].softmax(lane, E);
                float dot = 0.0f;
#pragma unroll
                for (int j = 0; j < X::NV; ++j)
#pragma unroll
                    for (int i = 0; i < X::VE; ++i) {
                        x[u].v[j][i] *= inv;
                        dot += x[u].v[j][i] * w[j][i];
                    }
                dot = join_lanes<L, LaneSum>(dot);
#pragma unroll
                for (int j = 0; j < X::NV; ++j)
#pragma unroll
                    for (int i = 0; i < X::VE; ++i)
                        x[u].v[j][i] = valid ? g * x[u].v[j][i] * (w[j][i] - dot) : 0.0f;
                x[u].store((char *)s.dlogits + row * E * T::size, lane, in ? E : 0);
            }
        }
    }
}

// f(T, L, N) of the logits' type and the number of experts.
template <class F>
const void *with_lanes(hoccl_dtype_t dt, int E, F &&f) {
    auto typed = [&](auto l, auto n) { return dt == HOCCL_BF16 ? f(EBF16(), l, n) : f(EF32(), l, n); };
#define HOCCL_LANES(l, n) return typed(std::integral_constant<int, l>(), std::integral_constant<int, n>())
    if (E > 512) HOCCL_LANES(64, 16);
    switch (lanes_of(E)) {
    case 1: HOCCL_LANES(1, 8);
    case 2: HOCCL_LANES(2, 8);
    case 4: HOCCL_LANES(4, 8);
    case 8: HOCCL_LANES(8, 8);
    case 16: HOCCL_LANES(16, 8);
    case 32: HOCCL_LANES(32, 8);
    }
    HOCCL_LANES(64, 8);
#undef HOCCL_LANES
}

// Workgroups of one batch, a pass each up to `most` of them.
uint32_t blocks_of(size_t tokens, int E, int threads, size_t most) {
    const size_t rows = (size_t)(threads / lanes_of(E) * kAhead), n = (tokens + rows - 1) / rows;
    return (uint32_t)(n < 1 ? 1 : n < most ? n : most);
}

}  // namespace

uint32_t balance_blocks(size_t tokens, int E, int batches) {
    return blocks_of(tokens, E, kThreads, batches <= 2 ? 256 : batches < 32 ? 512 / batches : 16);
}

hipError_t launch_balance(const BalanceArgs &a, hoccl_dtype_t dt, int wg, hipStream_t s) {
    const void *k = with_lanes(dt, a.E, [](auto t, auto l, auto n) {
        return (const void *)balance_kernel<decltype(t), decltype(l)::value, decltype(n)::value>;
    });
    void *args[] = {(void *)&a};
    return hipLaunchKernel(k, dim3((unsigned)wg), dim3(kThreads), args, 0, s);
}

hipError_t launch_balance_finish(const BalanceArgs &a, int wg, hipStream_t s) {
    void *args[] = {(void *)&a};
    return hipLaunchKernel((const void *)balance_finish_kernel, dim3((unsigned)wg), dim3(kFinishThreads), args, 0, s);
}

uint32_t balance_backward_blocks(size_t tokens, int E) { return blocks_of(tokens, E, kOpThreads, 4096); }

hipError_t launch_balance_backward(const BalanceArgs &a, hoccl_dtype_t dt, int wg, hipStream_t s) {
    const void *k = with_lanes(dt, a.E, [](auto t, auto l, auto n) {
        return (const void *)balance_backward_kernel<decltype(t), decltype(l)::value, decltype(n)::value>;
    });
    void *args[] = {(void *)&a};
    return hipLaunchKernel(k, dim3((unsigned)wg), dim3(kOpThreads), args, 0, s);
}

}  // namespace hoccl
