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
// L lanes hold a token's logits, 8 or 16 each (logits_of), in
// vectors of 16 bytes; two tokens of every lane are in flight.  The sums over
// tokens stay in registers and are joined once a workgroup; choices are
// counted in LDS, in integers, whose order does not matter.  The partial sums
// of the workgroups, a number that goes by the sizes alone, are added in order
// by one workgroup a batch.
//
// Memory's part is logits and choices read once and gradients written; the
// forward pass at many tokens has as much arithmetic, some 8 instructions a
// logit, and four waves a SIMD do not hide one behind the other (eight batches of
// 9,800 to 32,768 tokens, 256 experts, bf16: 25.4 us, where memory alone and
// arithmetic alone would take 15 each, and 6.5 for the sums' end; backward 29.4
// us for 180 MB).  At few tokens it is the launches and the latency of the last
// sum.
#include <algorithm>
#include <type_traits>

#include "lanes.h"
#include "shard_ops.h"

namespace hoccl {
namespace {

constexpr int kThreads = 512;  // of the forward pass's first kernel
constexpr int kWaves = kThreads / 64;
constexpr int kAhead = 2;      // tokens of a lane in flight
// Workgroups of the forward pass, and half of them at most for one batch: two a
// CU, which is what its registers hold (of fp32 over 512 experts one alone, so
// two rounds).  Every workgroup makes as many passes as the others, whatever the
// batches' lengths (eight batches of 9,800 to 32,768 tokens, 256 experts: 2 us
// less than with as many workgroups for each), and whole ones, so that places
// may stay empty (there 448 of 512 are taken).
constexpr size_t kBlocks = 512;
constexpr float kLog2e = 1.4426950408889634f;

// Logits of a lane.  16 leave fewer lanes to exchange with but more registers
// for fewer waves: forward, 8 x 16384 tokens and 256 experts take 15 % less with
// 16 than with 8 in bf16, but 28 % more in fp32, and of 128 experts 27 % more in
// bf16.
int logits_of(int E, hoccl_dtype_t dt, bool backward) {
    return E > 512 || (!backward && dt == HOCCL_BF16 && E > 128) ? 16 : 8;
}
int lanes_of(int E, int logits) {
    int l = 1;
    while (l < 64 && l * logits < E) l *= 2;
    return l;
}

// Batches of no more passes than this are a workgroup's each, which finishes
// its batch without a second kernel (and without a workspace).  A pass more
// costs that workgroup 1.4 to 2.2 us, and 3.8 where one lane counts all of a
// token's choices (up to 8 experts); the second kernel costs 3 us on the
// device and 3 to 4.5 more of an eager call, which waits for the host.  One
// batch forward, one kernel / two, replayed and eager, in us:
//
//   lanes, experts  passes  tokens  replayed      eager
//   1, 8            2       2048    13.6 / 13.9   14.4 / 16.3
//                   3       3072    17.4 / 14.1   18.3 / 17.8
//   2, 16           3       1536    13.3 / 11.5   14.2 / 17.7
//                   4       2048    16.1 / 11.7   16.9 / 17.9
//   4, 32           3       768     12.1 / 10.4   13.5 / 16.8
//                   4       1024    14.5 / 10.6   15.2 / 17.9
//   8, 64           4       512     10.0 /  9.0   13.5 / 17.7
//                   6       768     12.8 /  9.2   13.6 / 17.6
//   64, 1024        4       64      12.6 / 10.9   13.5 / 17.8
//                   6       96      16.4 / 11.1   17.2 / 17.8
//
// Up to the limits an eager call gains twice what a replayed one loses, or
// more; both go one way, as a replay has to have the eager call's bits.
size_t one_passes(int lanes) { return lanes < 2 ? 2 : lanes < 8 ? 3 : 4; }

// Choice i behind `experts`, -1 where it is no expert.
__device__ __forceinline__ int choice(const BalanceArgs &a, const char *experts, uint32_t i) {
    if (a.index64) {
        const uint64_t v = ((const uint64_t *)experts)[i];
        return v < (uint64_t)a.E ? (int)v : -1;
    }
    const uint32_t v = ((const uint32_t *)experts)[i];
    return v < (uint32_t)a.E ? (int)v : -1;
}

// f(choice) of a lane's choices but the first of a token whose `k` choices
// start at `at`: eight reads at once, since one after another each would wait
// for memory.
template <int L, class F>
__device__ __forceinline__ void more_choices(const BalanceArgs &a, const char *experts, uint32_t at, int lane, int k,
                                             F &&f) {
    constexpr int AHEAD = 8;
    for (int c = lane + L; c < k; c += AHEAD * L) {
        int e[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) e[i] = c + i * L < k ? choice(a, experts, at + c + i * L) : -1;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) f(e[i]);
    }
}

// A lane's logits of one token: NV vectors of VE, L lanes apart.
template <class T, int L, int N>
struct Logits {
    static constexpr int VE = 16 / T::size, NV = N / VE;
    // As they are read, and as numbers.
    struct Packed {
        Raw<16> v[NV];
        __device__ __forceinline__ void load(const void *p, int lane, int E) {
#pragma unroll
            for (int j = 0; j < NV; ++j) load_window<T>(p, at(j, lane), E, v[j]);
        }
    };
    float v[NV][VE];
    __device__ __forceinline__ Logits(Packed x, int lane, int E) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (E < L * N) settle_window<T>(at(j, lane), E, x.v[j]);
            T::template unpack<VE>(x.v[j], v[j]);
        }
    }
    static __device__ __forceinline__ int at(int j, int lane) { return (j * L + lane) * VE; }
    __device__ __forceinline__ void store(void *p, int lane, int E) const {
#pragma unroll
        for (int j = 0; j < NV; ++j) store_some<T, true>(p, at(j, lane), E, v[j]);
    }
    // To exp(x - max) over the L lanes; returns what makes them p: the
    // reciprocal of their sum, an approximation and a Newton step (half a step
    // off; all of a token's p carry it).  Behind E there are zeros.
    // log2 e is one fp32 number, 1.3e-8 of the exponents off: 64 logits of
    // deviation 3 have p with 7.8e-8 of rounding errors (relative, in the 2-norm), with
    // an exact one 7.3e-8 for two more instructions a logit of about eight.
    __device__ __forceinline__ float softmax(int lane, int E) {
        float top = -INFINITY, sum = 0.0f;
        if (E < L * N)
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int mine = here(E - at(j, lane));
#pragma unroll
                for (int i = 0; i < VE; ++i)
                    if (i >= mine) v[j][i] = -INFINITY;
            }
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VE; ++i) top = fmaxf(top, v[j][i]);
        top = join_lanes<L, LaneMax>(top);
        if (fabsf(top) <= 65536.0f) {
            // In one step; the rounding of top log2 e (2^-8 at most) is the
            // same factor for all and goes with the sum.
            const float base = -top * kLog2e;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VE; ++i) v[j][i] = __builtin_amdgcn_exp2f(fmaf(v[j][i], kLog2e, base));
        } else {
            // All -inf: -inf - 0 leaves p = 0.  Others as large: that factor
            // would leave fp32's range from 2^30 on.
            const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VE; ++i) v[j][i] = __builtin_amdgcn_exp2f((v[j][i] - base) * kLog2e);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VE; ++i) sum += v[j][i];
        sum = join_lanes<L, LaneSum>(sum);
        const float inv = __builtin_amdgcn_rcpf(sum);
        return sum == 0.0f ? 0.0f : fmaf(fmaf(-sum, inv, 1.0f), inv, inv);
    }
};

// Whether any of the L lanes of this lane's group has `v`.
template <int L>
__device__ __forceinline__ bool any_lane(bool v) {
    const uint64_t all = __ballot(v);
    if constexpr (L == 64) return all != 0;
    const uint32_t lane = threadIdx.x % 64;
    return (all >> (lane / L * L) & ((1ull << L % 64) - 1)) != 0;
}

// The batch of a block, and its place among the batch's blocks.
__device__ __forceinline__ int batch_of(const BalanceArgs &a, uint32_t block, uint32_t &lb, uint32_t &nb) {
    int seg = 0;
    while (a.first[seg + 1] <= block) ++seg;
    nb = a.first[seg + 1] - a.first[seg], lb = block - a.first[seg];
    return seg;
}

// Loss, weights and counts of a batch from its sums: the table's columns, in
// 64 bits.  For all threads of a workgroup of NT.
template <int NT>
__device__ __forceinline__ void finish_batch(const BalanceArgs &a, int seg, const double *tot) {
    constexpr int OWN = (kMaxExperts + NT - 1) / NT;  // experts of a thread
    __shared__ int rank_choices[64];
    __shared__ double red[NT / 64][2];
    const int E = a.E, D = a.D, per = E / D, t = threadIdx.x;
    for (int e = t; e < E; e += NT) a.expert_tokens[(uint64_t)seg * E + e] = (int32_t)tot[E + e];
    if (t < D) a.rank_tokens[(uint64_t)seg * D + t] = (int32_t)tot[2 * E + t];
    for (int d = t / 64; d < D; d += NT / 64) {  // a wave a rank
        int n = 0;
        for (int e = d * per + t % 64; e < (d + 1) * per; e += 64) n += (int)tot[E + e];
        n = join_lanes<64, LaneSum>(n);
        if (t % 64 == 0) rank_choices[d] = n;
    }
    __syncthreads();
    const double live = tot[2 * E + D], over = live > 0.0 ? 1.0 / live : 0.0;
    double loss = 0.0, all = 0.0, w[OWN] = {};
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int e = i * NT + t;
        if (e >= E) continue;
        const int d = (int)(((uint32_t)e * a.rank_mul) >> 21);
        w[i] = (a.expert_scale * tot[E + e] + a.rank_scale * rank_choices[d] + a.traffic_scale * tot[2 * E + d]) * over;
        loss += w[i] * tot[e] * over;
        all += w[i];
    }
    loss = join_lanes<64, LaneSum>(loss);
    all = join_lanes<64, LaneSum>(all);
    if (t % 64 == 0) red[t / 64][0] = loss, red[t / 64][1] = all;
    __syncthreads();
    loss = 0.0, all = 0.0;
    for (int i = 0; i < min((E + 63) / 64, NT / 64); ++i) loss += red[i][0], all += red[i][1];
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int e = i * NT + t;
        if (e < E) a.coef[(uint64_t)seg * E + e] = (float)((w[i] - all / E) * over);
    }
    if (t == 0) a.loss[seg] = (float)loss;
    __syncthreads();
}

constexpr int kColumns = 2 * kMaxExperts + 64 + 4;

// ONE: every batch is one workgroup's, which finishes it.
template <class T, int L, int N, bool ONE>
__global__ void __launch_bounds__(kThreads) balance_kernel(BalanceArgs) {
    const BalanceArgs &a = kernel_args<BalanceArgs>();
    using X = Logits<T, L, N>;
    constexpr int ROWS = kThreads / L;     // tokens of a workgroup's pass, kAhead times
    constexpr int OWN = 64 / L < N ? 64 / L : N;  // ranks a lane counts: its experts at most, 64 in all
    __shared__ float sum_p[kWaves][L * N];
    // Choices, a copy for each of a wave's groups, so that the 64 lanes that
    // hold tokens of 8 experts do not meet at eight addresses.
    constexpr int COPIES = 64 / L;
    __shared__ int sum_n[L * N * COPIES];
    __shared__ int sum_sent[64];
    __shared__ int sum_live;
    __shared__ double tot[ONE ? kColumns : 1];
    const int E = a.E, D = a.D, k = a.k, stride = balance_columns(E, D);
    if constexpr (L > 1) __builtin_assume(E > N);  // over the logits of one lane
    const int lane = threadIdx.x % L, slot = threadIdx.x / L;
    for (uint32_t block = blockIdx.x; block < a.first[a.nseg]; block += gridDim.x) {
        uint32_t lb, nb;
        const int seg = batch_of(a, block, lb, nb);
        const BalanceSeg &s = a.seg[seg];
        for (int e = threadIdx.x; e < E * COPIES; e += kThreads) sum_n[e] = 0;
        if (threadIdx.x < 64) sum_sent[threadIdx.x] = 0;
        if (threadIdx.x == 0) sum_live = 0;
        __syncthreads();
        float acc[X::NV][X::VE] = {};
        int sent[OWN] = {}, live = 0;
        // What a pass reads is loaded during the pass before it.
        typename X::Packed next[kAhead];
        int next_first[kAhead];  // the lane's first choice of each token
        auto load = [&](uint64_t row0) {
            const char *logits = (const char *)s.logits + row0 * E * T::size;
            const char *experts = (const char *)s.experts + row0 * k * (a.index64 ? 8 : 4);
            const uint64_t left = s.tokens - row0;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                // A row behind the last reads the pass's first instead and,
                // without choices, is padding.
                const uint32_t row = u * ROWS + slot;
                const bool in = row < left;
                next[u].load(logits + (in ? row : 0) * (uint32_t)E * T::size, lane, E);
                next_first[u] = in && lane < k ? choice(a, experts, row * k + lane) : -1;
            }
        };
        const uint64_t step = (uint64_t)nb * ROWS * kAhead;
        uint64_t row0 = (uint64_t)lb * ROWS * kAhead;
        if (row0 < s.tokens) load(row0);
        for (; row0 < s.tokens; row0 += step) {
            typename X::Packed now[kAhead];
            int first[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) now[u] = next[u], first[u] = next_first[u];
            if (row0 + step < s.tokens) load(row0 + step);
            const char *experts = (const char *)s.experts + row0 * k * (a.index64 ? 8 : 4);
            const uint64_t left = s.tokens - row0;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint32_t row = u * ROWS + slot;
                uint32_t lo = 0, hi = 0;  // the ranks that the token goes to
                auto choose = [&](int e) {
                    if (e < 0) return;
                    const uint32_t d = ((uint32_t)e * a.rank_mul) >> 21;
                    if (d < 32) lo |= 1u << d;
                    else hi |= 1u << (d - 32);
                    atomicAdd(&sum_n[e * COPIES + slot % COPIES], 1);
                };
                choose(first[u]);
                more_choices<L>(a, experts, row * k, lane, row < left ? k : 0, choose);
                lo = join_lanes<L, LaneOr>(lo);
                if (D > 32) hi = join_lanes<L, LaneOr>(hi);
                if ((lo | hi) == 0) continue;  // padding, for all of the token's lanes
                if (lane == 0) ++live;
#pragma unroll
                for (int i = 0; i < OWN; ++i) {
                    const int d = i * L + lane;
                    sent[i] += ((d < 32 ? lo : hi) >> (d & 31)) & 1u;
                }
                X x(now[u], lane, E);
                const float inv = x.softmax(lane, E);
#pragma unroll
                for (int j = 0; j < X::NV; ++j)
#pragma unroll
                    for (int i = 0; i < X::VE; ++i) acc[j][i] += x.v[j][i] * inv;
            }
        }
        // The wave's groups, then the waves: sums of p in order.
#pragma unroll
        for (int j = 0; j < X::NV; ++j)
#pragma unroll
            for (int i = 0; i < X::VE; ++i) acc[j][i] = join_groups<L, LaneSum>(acc[j][i]);
#pragma unroll
        for (int i = 0; i < OWN; ++i) sent[i] = join_groups<L, LaneSum>(sent[i]);
        live = join_groups<L, LaneSum>(live);
        if (threadIdx.x % 64 < L) {
#pragma unroll
            for (int j = 0; j < X::NV; ++j)
#pragma unroll
                for (int i = 0; i < X::VE; ++i) sum_p[threadIdx.x / 64][X::at(j, lane) + i] = acc[j][i];
#pragma unroll
            for (int i = 0; i < OWN; ++i)
                if (sent[i]) atomicAdd(&sum_sent[i * L + lane], sent[i]);
            if (live) atomicAdd(&sum_live, live);
        }
        __syncthreads();
        int32_t *out = a.partial + (uint64_t)block * stride;
        for (int e = threadIdx.x; e < E; e += kThreads) {
            float p = 0.0f;
            int n = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) p += sum_p[w][e];
#pragma unroll 8
            for (int c = 0; c < COPIES; ++c) n += sum_n[e * COPIES + c];
            if constexpr (ONE) tot[e] = p, tot[E + e] = n;
            else out[e] = __float_as_int(p), out[E + e] = n;
        }
        if constexpr (ONE) {
            if ((int)threadIdx.x < D) tot[2 * E + threadIdx.x] = sum_sent[threadIdx.x];
            if (threadIdx.x == 0) tot[2 * E + D] = sum_live;
            __syncthreads();
            finish_batch<kThreads>(a, seg, tot);
        } else {
            if ((int)threadIdx.x < D) out[2 * E + threadIdx.x] = sum_sent[threadIdx.x];
            if (threadIdx.x == 0) out[2 * E + D] = sum_live;
            __syncthreads();
        }
    }
}

// The same from the sums of a batch's blocks, rows of the table.  Lots of rows
// are added side by side, four columns a thread and twelve rows of them in
// flight, then the lots in order: 6.5 us, all latency (one row and column after
// another took four times as long, a column a thread 1.4 times, for 64 blocks of
// 256 experts).
constexpr int kFinishThreads = 1024;
constexpr int kLotAhead = 12;
__global__ void __launch_bounds__(kFinishThreads) balance_finish_kernel(BalanceArgs) {
    const BalanceArgs &a = kernel_args<BalanceArgs>();
    __shared__ double lot[kFinishThreads][4];
    __shared__ double tot[kColumns];
    const int E = a.E, cols = balance_columns(E, a.D), t = threadIdx.x;
    const int wide = cols / 4, lots = kFinishThreads / wide, g = t / wide, c = t % wide * 4;
    for (int seg = blockIdx.x; seg < a.nseg; seg += gridDim.x) {
        const uint32_t nb = a.first[seg + 1] - a.first[seg];
        const int32_t *rows = a.partial + (uint64_t)a.first[seg] * cols + c;
        if (g < lots) {
            double sum[4] = {};
            for (uint32_t b0 = g; b0 < nb; b0 += kLotAhead * lots) {
                Raw<16> v[kLotAhead];
#pragma unroll
                for (int i = 0; i < kLotAhead; ++i) {
                    const uint32_t b = b0 + i * lots;
                    if (b < nb) load_raw(v[i], rows + (uint64_t)b * cols);
                    else v[i] = {};
                }
#pragma unroll
                for (int i = 0; i < kLotAhead; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        sum[j] += c + j < E ? (double)__uint_as_float(v[i].w[j]) : (double)(int32_t)v[i].w[j];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) lot[t][j] = sum[j];
        }
        __syncthreads();
        for (int i = t; i < cols; i += kFinishThreads) {
            double sum = 0.0;
#pragma unroll 8
            for (int l = 0; l < lots; ++l) sum += lot[l * wide + i / 4][i % 4];
            tot[i] = sum;
        }
        __syncthreads();
        finish_batch<kFinishThreads>(a, seg, tot);
    }
}

template <class T, int L, int N>
__global__ void __launch_bounds__(kOpThreads) balance_backward_kernel(BalanceArgs) {
    const BalanceArgs &a = kernel_args<BalanceArgs>();
    using X = Logits<T, L, N>;
    constexpr int ROWS = kOpThreads / L;
    const int E = a.E, k = a.k;
    if constexpr (L > 1) __builtin_assume(E > N);  // over the logits of one lane
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
            const char *logits = (const char *)s.logits + row0 * E * T::size;
            const char *experts = (const char *)s.experts + row0 * k * (a.index64 ? 8 : 4);
            char *dlogits = (char *)s.dlogits + row0 * E * T::size;
            const uint64_t left = s.tokens - row0;
            typename X::Packed now[kAhead];
            bool any[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint32_t row = u * ROWS + slot;
                const bool in = row < left;
                now[u].load(logits + (in ? row : 0) * (uint32_t)E * T::size, lane, E);
                any[u] = in && lane < k && choice(a, experts, row * k + lane) >= 0;
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint32_t row = u * ROWS + slot;
                const bool in = row < left;
                more_choices<L>(a, experts, row * k, lane, in ? k : 0, [&](int e) { any[u] |= e >= 0; });
                X x(now[u], lane, E);
                if (any_lane<L>(any[u])) {
                    const float inv = x.softmax(lane, E), scale = g * inv;
                    float dot = 0.0f;
#pragma unroll
                    for (int j = 0; j < X::NV; ++j)
#pragma unroll
                        for (int i = 0; i < X::VE; ++i) dot += x.v[j][i] * w[j][i];
                    const float mean = join_lanes<L, LaneSum>(dot) * inv * scale;
#pragma unroll
                    for (int j = 0; j < X::NV; ++j)
#pragma unroll
                        for (int i = 0; i < X::VE; ++i) x.v[j][i] *= fmaf(w[j][i], scale, -mean);
                } else {
#pragma unroll
                    for (int j = 0; j < X::NV; ++j)
#pragma unroll
                        for (int i = 0; i < X::VE; ++i) x.v[j][i] = 0.0f;
                }
                x.store(dlogits + row * (uint32_t)E * T::size, lane, in ? E : 0);
            }
        }
    }
}

// f(T, L, N) of the logits' type and the number of experts.
template <bool BACKWARD, class F>
const void *with_lanes(hoccl_dtype_t dt, int E, F &&f) {
    const int n = logits_of(E, dt, BACKWARD), l = lanes_of(E, n);
    auto typed = [&](auto l, auto n) { return dt == HOCCL_BF16 ? f(EBF16(), l, n) : f(EF32(), l, n); };
#define HOCCL_LANES(l, n) return typed(std::integral_constant<int, l>(), std::integral_constant<int, n>())
    if (n == 16 && l == 64) HOCCL_LANES(64, 16);
    using std::integral_constant;
    if constexpr (!BACKWARD) {  // over 128 experts bf16 has 16 logits a lane, fp32 8
        if (n == 16 && l == 32) return f(EBF16(), integral_constant<int, 32>(), integral_constant<int, 16>());
        if (n == 16) return f(EBF16(), integral_constant<int, 16>(), integral_constant<int, 16>());
        if (l == 32) return f(EF32(), integral_constant<int, 32>(), integral_constant<int, 8>());
        if (l == 64) return f(EF32(), integral_constant<int, 64>(), integral_constant<int, 8>());
    } else {
        if (l == 32) HOCCL_LANES(32, 8);
        if (l == 64) HOCCL_LANES(64, 8);
    }
    switch (l) {
    case 1: HOCCL_LANES(1, 8);
    case 2: HOCCL_LANES(2, 8);
    case 4: HOCCL_LANES(4, 8);
    case 8: HOCCL_LANES(8, 8);
    }
    HOCCL_LANES(16, 8);
#undef HOCCL_LANES
}

size_t rows_of(int threads, int lanes) { return (size_t)(threads / lanes * kAhead); }
size_t over(size_t n, size_t d) { return (n + d - 1) / d; }

}  // namespace

void balance_blocks(const size_t *tokens, int E, hoccl_dtype_t dt, int batches, uint32_t *first) {
    const int lanes = lanes_of(E, logits_of(E, dt, false));
    const size_t rows = rows_of(kThreads, lanes);
    size_t all = 0, longest = 0;
    for (int b = 0; b < batches; ++b) all += over(tokens[b], rows), longest = std::max(longest, tokens[b]);
    first[0] = 0;
    if (longest <= rows * one_passes(lanes)) {
        for (int b = 0; b < batches; ++b) first[b + 1] = (uint32_t)(b + 1);
        return;
    }
    const size_t passes = std::max({(size_t)1, over(all, kBlocks), over(over(longest, rows), kBlocks / 2)});
    for (int b = 0; b < batches; ++b)
        first[b + 1] = first[b] + (uint32_t)std::max((size_t)1, over(tokens[b], rows * passes));
}

hipError_t launch_balance(const BalanceArgs &a, hoccl_dtype_t dt, int wg, hipStream_t s) {
    const bool one = balance_is_one(a.first, a.nseg);
    const void *k = with_lanes<false>(dt, a.E, [&](auto t, auto l, auto n) {
        constexpr int L = decltype(l)::value, N = decltype(n)::value;
        return one ? (const void *)balance_kernel<decltype(t), L, N, true>
                   : (const void *)balance_kernel<decltype(t), L, N, false>;
    });
    void *args[] = {(void *)&a};
    return hipLaunchKernel(k, dim3((unsigned)wg), dim3(kThreads), args, 0, s);
}

hipError_t launch_balance_finish(const BalanceArgs &a, int wg, hipStream_t s) {
    void *args[] = {(void *)&a};
    return hipLaunchKernel((const void *)balance_finish_kernel, dim3((unsigned)wg), dim3(kFinishThreads), args, 0, s);
}

uint32_t balance_backward_blocks(size_t tokens, int E, hoccl_dtype_t dt) {
    const size_t rows = rows_of(kOpThreads, lanes_of(E, logits_of(E, dt, true)));
    return (uint32_t)std::min((size_t)4096, std::max((size_t)1, over(tokens, rows)));
}

hipError_t launch_balance_backward(const BalanceArgs &a, hoccl_dtype_t dt, int wg, hipStream_t s) {
    const void *k = with_lanes<true>(dt, a.E, [](auto t, auto l, auto n) {
        return (const void *)balance_backward_kernel<decltype(t), decltype(l)::value, decltype(n)::value>;
    });
    void *args[] = {(void *)&a};
    return hipLaunchKernel(k, dim3((unsigned)wg), dim3(kOpThreads), args, 0, s);
}

}  // namespace hoccl
