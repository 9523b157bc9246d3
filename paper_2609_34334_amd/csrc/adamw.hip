// AdamW over many tensors in one launch, states in 32 or 8 bits.
//
//   g  = grad * grad_scale
//   m' = beta1 m + (1 - beta1) g        v' = beta2 v + (1 - beta2) g g
//   p' = (1 - lr wd) p - lr / (1 - beta1^t) m' / (sqrt(v') / sqrt(1 - beta2^t) + eps)
//
// and, where a copy is asked for, bf16(p'): what the all-gather of the
// parameters sends out.  All arithmetic is in fp32, whatever is stored.
//
// 8-bit states: a block of 128 elements of a tensor keeps m' as e4m3 values
// and their fp32 scale (largest magnitude over 448), and v' as sqrt(v') in
// the same form, which halves the range that v' spans.  m' and v' are
// rounded only after the update has used them.  A root that is not zero is
// never stored as zero (2^-9 of the scale at least): the next step divides
// by it.
//
// The states' products and sums are written without fused multiply-adds,
// and sqrt and the scales' divisions are correctly rounded, so that the
// states are those of the formulas taken one operation at a time in fp32.
//
// Bound by memory: 28 bytes an element (fp32 parameters and states, bf16
// gradients and copies; 25.2M elements in 117 us, 6.0 TB/s), 16.1 with 8-bit
// states (62 us, 6.5 TB/s, part of it from the caches).  Many small tensors
// are bound by the launches, of kAdamSegs tensors each, and by the host.
#include <algorithm>
#include <type_traits>

#include "lanes.h"
#include "shard_ops.h"

#pragma clang fp contract(off)

namespace hoccl {
namespace {

// Elements of a lane's vector, and vectors of a thread in a tile.  With 25.2M
// elements two vectors of four take 4 % longer than one in 32 bits, and 6 % less
// in 8 bits, where two share the work on their scales.  With bf16 parameters
// one of eight makes wider accesses: 6 % less, but 10 % more with fp32 ones,
// whose 32 bytes a lane are two accesses with gaps.
template <class TP, bool Q8>
constexpr int kVE = Q8 && TP::size == 2 ? 8 : 4;
template <class TP, bool Q8>
constexpr int kU = Q8 ? 8 / kVE<TP, Q8> : 1;
template <bool Q8>
constexpr uint32_t kTile = kOpThreads * (Q8 ? 8 : 4);

// Every byte is used once a step: reads and writes are non-temporal (25.2M
// elements, 32 bits: plain ones take 14 % longer).  The codes of 8-bit states,
// four bytes a lane, are plain (non-temporal 4 % longer).
constexpr bool kNT = true;

struct Hyper {
    float b1, c1, b2, c2, decay, rate, root, eps, gs;
};

// New moments of one element, and its parameter.
__device__ __forceinline__ float step_one(const Hyper &h, float p, float g, float &m, float &v, float &r) {
    g = g * h.gs;
    m = m * h.b1 + g * h.c1;
    v = v * h.b2 + g * g * h.c2;
    r = __builtin_sqrtf(v);
    // The reciprocal (1 ulp) instead of a division, whose 11 instructions 25.2M
    // elements of 8-bit states felt: 6 % longer.  The update's error hardly
    // shows in the parameter, which is larger by far.  The divisor is
    // zero or normal (eps is, and the smallest root is 2^-75).
    return p * h.decay - h.rate * m * __builtin_amdgcn_rcpf(r * h.root + h.eps);
}

template <class T, bool NT, bool FULL, int B>
__device__ __forceinline__ void load(const void *p, uint64_t e, uint64_t n, Raw<B> &r) {
    if constexpr (FULL) load_raw<NT>(r, (const char *)p + e * T::size);
    else load_window<T, NT>(p, e, n, r);
}
template <class T, bool FULL, int VE>
__device__ __forceinline__ void store(void *p, uint64_t e, uint64_t n, const float (&f)[VE]) {
    if constexpr (FULL) {
        Raw<T::size * VE> r;
        T::template pack<VE>(f, r);
        store_raw<kNT>((char *)p + e * T::size, r);
    } else {
        store_some<T, kNT>(p, e, n, f);
    }
}

// The vectors' moments as e4m3 bytes and scales.  The blocks that a block's
// lanes hold (m and the root of v, once or twice) share the divisions for their
// scales: of neighbouring lanes each makes those of one block and gives the
// result to the others.
template <bool FULL, int U, int VE>
__device__ __forceinline__ void put_blocks(const AdamTensor &s, uint64_t base, uint64_t n, const float (&m)[U][VE],
                                           const float (&r)[U][VE]) {
    constexpr int L = kBlock / VE, N = 2 * U;
    const uint32_t q = threadIdx.x % N;
    uint32_t top[N];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        top[2 * u] = join_lanes<L, LaneUMax>(top_bits(m[u]));
        top[2 * u + 1] = join_lanes<L, LaneUMax>(top_bits(r[u]));
    }
    float scale, mine, inv[N];
    if constexpr (U == 2) {
        block_scale(__uint_as_float(q < 2 ? (q == 0 ? top[0] : top[1]) : (q == 2 ? top[2] : top[3])), scale, mine);
        inv[0] = dpp<0x00>(mine), inv[1] = dpp<0x55>(mine), inv[2] = dpp<0xAA>(mine), inv[3] = dpp<0xFF>(mine);
    } else {
        block_scale(__uint_as_float(q == 0 ? top[0] : top[1]), scale, mine);
        inv[0] = dpp<0xA0>(mine), inv[1] = dpp<0xF5>(mine);  // quad_perm 0,0,2,2 and 1,1,3,3
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint64_t e = base + (uint64_t)(u * kOpThreads + threadIdx.x) * VE;
        float x[VE], y[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            x[i] = m[u][i] * inv[2 * u];
            y[i] = r[u][i] * inv[2 * u + 1];
            // A root that is not zero is not held as zero.
            y[i] = y[i] > 0.0f && y[i] < kLeast ? kLeast : y[i];
        }
        Raw<VE> a, b;
        to_e4m3(x, a);
        to_e4m3(y, b);
        if constexpr (FULL) {
            store_raw((char *)s.m + e, a);
            store_raw((char *)s.v + e, b);
        } else {
            store_bytes(s.m, e, n, a);
            store_bytes(s.v, e, n, b);
        }
    }
    const uint64_t first = base + (uint64_t)(q / 2 * kOpThreads + threadIdx.x / L * L) * VE;
    if (threadIdx.x % L < N && (FULL || first < n)) (q % 2 ? s.v_scale : s.m_scale)[first / kBlock] = scale;
}

// FULL: the tile ends before the tensor does.
template <class TP, class TG, bool Q8, bool FULL>
__device__ __forceinline__ void tile(const AdamTensor &s, const Hyper &h, uint64_t base) {
    constexpr int U = kU<TP, Q8>, VE = kVE<TP, Q8>;
    const uint64_t n = FULL ? base + kTile<Q8> : s.n;
    float p[U][VE], g[U][VE], m[U][VE], v[U][VE];
    using TS = std::conditional_t<Q8, EByte, EF32>;
    Raw<TP::size * VE> rp[U];
    Raw<TG::size * VE> rg[U];
    Raw<TS::size * VE> rm[U], rv[U];
    float sm[U], sv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint64_t e = base + (uint64_t)(u * kOpThreads + threadIdx.x) * VE;
        load<TP, kNT, FULL>(s.param, e, n, rp[u]);
        load<TG, kNT, FULL>(s.grad, e, n, rg[u]);
        load<TS, kNT && !Q8, FULL>(s.m, e, n, rm[u]);
        load<TS, kNT && !Q8, FULL>(s.v, e, n, rv[u]);
        if constexpr (Q8) {
            const uint64_t block = (FULL || e < n ? e : n - 1) / kBlock;
            sm[u] = s.m_scale[block], sv[u] = s.v_scale[block];
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint64_t e = base + (uint64_t)(u * kOpThreads + threadIdx.x) * VE;
        if constexpr (!FULL) {
            settle_window<TP>(e, n, rp[u]);
            settle_window<TG>(e, n, rg[u]);
            settle_window<TS>(e, n, rm[u]);
            settle_window<TS>(e, n, rv[u]);
        }
        TP::template unpack<VE>(rp[u], p[u]);
        TG::template unpack<VE>(rg[u], g[u]);
        if constexpr (Q8) {
            from_e4m3(rm[u], m[u]);
            from_e4m3(rv[u], v[u]);
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                m[u][i] *= sm[u];
                const float r = v[u][i] * sv[u];
                v[u][i] = r * r;
            }
        } else {
            EF32::unpack<VE>(rm[u], m[u]);
            EF32::unpack<VE>(rv[u], v[u]);
        }
    }
    float r[U][VE];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint64_t e = base + (uint64_t)(u * kOpThreads + threadIdx.x) * VE;
#pragma unroll
        for (int i = 0; i < VE; ++i) p[u][i] = step_one(h, p[u][i], g[u][i], m[u][i], v[u][i], r[u][i]);
        if constexpr (!Q8) {
            store<EF32, FULL>(s.m, e, n, m[u]);
            store<EF32, FULL>(s.v, e, n, v[u]);
        }
        store<TP, FULL>(s.param, e, n, p[u]);
        if (s.copy) store<EBF16, FULL>(s.copy, e, n, p[u]);
    }
    // Behind the end m and v are zero: nothing there is the largest of a block.
    if constexpr (Q8) put_blocks<FULL>(s, base, n, m, r);
}

__device__ __forceinline__ AdamTensor tensor_of(const AdamSeg &s) {
    auto word = [&](int i) { return (uint64_t)(s.hi[i / 2] >> i % 2 * 16 & 0xffff) << 32 | s.lo[i]; };
    return {(void *)word(0),  (const void *)word(1), (void *)word(2), (void *)word(3),
            (float *)word(4), (float *)word(5),      (void *)word(6), word(7)};
}

template <class TP, class TG, bool Q8, int CAP>
__global__ void __launch_bounds__(kOpThreads) adamw_kernel(AdamArgsT<CAP>) {
    const AdamArgsT<CAP> &a = kernel_args<AdamArgsT<CAP>>();
    const AdamStep &c = a.step;
    Hyper h = {c.b1, c.c1, c.b2, c.c2, c.decay, c.rate, c.root, c.eps, c.grad_scale ? *c.grad_scale : 1.0f};
    if (c.lr_dev || c.t_dev) {
        // 1 - beta^t in 64 bits: in 32 the difference of the first steps
        // would keep four digits.
        const double lr = c.lr_dev ? (double)*c.lr_dev : c.lr;
        const double t = c.t_dev ? fmax(1.0, (double)*c.t_dev) : c.t;
        h.decay = (float)(1.0 - lr * c.weight_decay);
        h.rate = (float)(lr / -expm1(t * c.log_b1));
        h.root = (float)(1.0 / sqrt(-expm1(t * c.log_b2)));
    }
    const uint32_t tiles = a.first[a.nseg];
    for (uint32_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        // Lane i looks at tensors i and 64 + i: one read of the table, where a
        // search would wait for six.
        int seg = -1;
#pragma unroll
        for (uint32_t part = 0; part < CAP; part += 64) {
            const uint32_t i = part + threadIdx.x % 64;
            seg += __popcll(__ballot(i < (uint32_t)a.nseg && a.first[i < CAP ? i : 0] <= t));
        }
        const AdamTensor s = tensor_of(a.seg[seg]);
        const uint64_t base = (uint64_t)(t - a.first[seg]) * kTile<Q8>;
        if (s.n - base >= kTile<Q8>) tile<TP, TG, Q8, true>(s, h, base);
        else tile<TP, TG, Q8, false>(s, h, base);
    }
}

template <int CAP>
hipError_t launch(const AdamArgsT<CAP> &a, hoccl_dtype_t param, hoccl_dtype_t grad, int bits, int wg, hipStream_t s) {
    const bool pb = param == HOCCL_BF16, gb = grad == HOCCL_BF16, q = bits == 8;
    const void *k;
    if (pb)
        k = gb ? (q ? (const void *)adamw_kernel<EBF16, EBF16, true, CAP>
                    : (const void *)adamw_kernel<EBF16, EBF16, false, CAP>)
               : (q ? (const void *)adamw_kernel<EBF16, EF32, true, CAP>
                    : (const void *)adamw_kernel<EBF16, EF32, false, CAP>);
    else
        k = gb ? (q ? (const void *)adamw_kernel<EF32, EBF16, true, CAP>
                    : (const void *)adamw_kernel<EF32, EBF16, false, CAP>)
               : (q ? (const void *)adamw_kernel<EF32, EF32, true, CAP>
                    : (const void *)adamw_kernel<EF32, EF32, false, CAP>);
    void *args[] = {(void *)&a};
    return hipLaunchKernel(k, dim3((unsigned)wg), dim3(kOpThreads), args, 0, s);
}

}  // namespace

uint32_t adamw_tile(int state_bits) { return state_bits == 8 ? kTile<true> : kTile<false>; }

hipError_t launch_adamw(const AdamArgs &a, hoccl_dtype_t param, hoccl_dtype_t grad, int state_bits, int wg,
                        hipStream_t s) {
    if (a.nseg > kAdamFewSegs) return launch(a, param, grad, state_bits, wg, s);
    // Few tensors pass a smaller struct, which the runtime stages faster.
    AdamArgsT<kAdamFewSegs> f;
    std::copy(a.seg, a.seg + a.nseg, f.seg);
    std::copy(a.first, a.first + a.nseg + 1, f.first);
    f.nseg = a.nseg;
    f.step = a.step;
    return launch(f, param, grad, state_bits, wg, s);
}

}  // namespace hoccl
