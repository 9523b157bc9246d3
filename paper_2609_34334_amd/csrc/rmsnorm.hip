// The residual's addition and the root-mean-square norm of its rows, and
// their gradients.
//
//   h = x + residual, rounded to their type        (h = x without a residual)
//   y = h w / sqrt(mean(h h) + eps)
//
// y is stored in the type of x, or in 8 bits: e4m3 values with an fp32 scale
// for each 128 of a row.  With u = h / sqrt(mean(h h) + eps) and the
// gradient dy of y, the sums over a row's elements,
//
//   dx = (dy w - u mean(dy w u)) / sqrt(mean(h h) + eps) + dres
//   dw = sum over the rows of dy u
//
// where dres is the gradient that h has from elsewhere.  dx is the gradient
// of x and of the residual.
//
// One pass over the data: a workgroup's threads (or a wave's: 64 vectors take
// one wave, with no exchange through LDS) hold a row in registers, a vector
// of 16 bytes each up to 1024 of them, so that what is read is read once.  The
// next row's reads are under way while a row is summed and written.  One
// vector a thread keeps the registers few and the waves many: up to four (256
// threads for 4096 elements, one wave for 2048), without the reads ahead, cost
// 23 % at 8192 x 4096, 38 % into 8 bits at 4096 x 2048 and 40 % in the gradients
// at 16384 x 4096.  Sums are in fp32, in an order that goes by the row's length
// alone.
//
// Where rows fill their last vectors the backward pass reads and writes past
// the caches (16384 x 4096: 12 % longer otherwise).  The forward pass writes
// past them (8 % longer otherwise at 4096 x 2048 into 8 bits, 2 % at 8192 x
// 4096); it reads through them where its inputs may still be there, past them
// in large calls (kFarBytes).
//
// Bound by memory: 8 bytes an element (bf16 with a residual: 42 us, 6.4 TB/s at
// 8192 x 4096), 7 with y in 8 bits (11.5 us, 5.1 TB/s at 4096 x 2048, two rows a
// workgroup); backward 8 bytes and the partial sums of the weight's gradient (82
// and 5 us, 6.2 TB/s, at 16384 x 4096).
#include <algorithm>
#include <type_traits>

#include "lanes.h"
#include "shard_ops.h"

namespace hoccl {
namespace {

template <class T>
constexpr int kVE = 16 / T::size;  // elements of a vector

// N weights from element e on, zeros at and behind H.
template <int N>
__device__ __forceinline__ void load_weights(const void *w, int bf16, uint32_t e, uint32_t H, float (&f)[N]) {
    if (bf16) load_some<EBF16>(w, e, H, f);
    else load_some<EF32>(w, e, H, f);
}

// What a thread holds of a row: NV vectors.  FULL: the vectors of the row's
// threads end where it does (checking for it in the loop costs the gradients at
// 16384 x 4096 6 %).
template <class T, int NV, bool FULL>
struct Shaped {
    static constexpr int VE = kVE<T>, N = NV * VE;
    // Longer rows (over 8192 bf16 elements) have no registers for the next
    // one; the longest none for the weights, which they read again, nor, in the
    // backward pass, for the residual's gradient, which is read last, and the
    // weights' gradients, which stay in LDS (rows of 20000 bf16 take 2.2 times as
    // long otherwise; but rows of 12288 fp32, whose 16 elements a thread fit, 17 %
    // longer so).
    static constexpr bool ahead = N <= 8, lean = N >= 32, keep_weights = N <= 16;
    // The offsets of many vectors, their comparisons with the row's end and their
    // addresses would be kept over the loop, in more registers than the row: they
    // are made anew for every row (20000 fp32: 2.7 times as long otherwise, the
    // gradients 1.6 times), of the longest again after its sums (16 % and 43 %
    // less).  The gradients of 8193 to 16384 elements whose last vectors are not
    // whole still keep 20 bytes of them a lane in scratch memory (bf16), 8 (fp32).
    static constexpr bool anew = NV >= 4, again = NV >= 8;
    Raw<16> v[NV];
    // W threads a row, of which this is number t.
    // Lines that two rows or two vectors share are read twice: through the
    // caches, whatever NT says (past them the gradients of 5003 bf16 take 27 %
    // longer, the norm of 2049 25 %).
    template <bool NT>
    __device__ __forceinline__ void load(const void *p, uint64_t row, uint32_t H, uint32_t W, uint32_t t) {
        const char *at = (const char *)p + row * H * T::size;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t e = (j * W + t) * VE;
            if constexpr (FULL) load_raw<NT>(v[j], at + e * T::size);
            else load_window<T>(at, e, H, v[j]);
        }
    }
    __device__ __forceinline__ void settle(uint32_t H, uint32_t W, uint32_t t) {
        if constexpr (!FULL)
#pragma unroll
        for (int j = 0; j < NV; ++j) settle_window<T>((j * W + t) * VE, H, v[j]);
    }
    __device__ __forceinline__ void unpack(int j, float (&f)[VE]) const { T::template unpack<VE>(v[j], f); }
    static __device__ __forceinline__ void store(void *p, uint32_t e, uint32_t H, const float (&f)[VE]) {
        if constexpr (FULL) {
            Raw<16> r;
            T::template pack<VE>(f, r);
            store_raw<true>((char *)p + e * T::size, r);
        } else {
            store_some<T, true>(p, e, H, f);
        }
    }
    // The same values, which the compiler takes for others: what it unpacked
    // before need not stay in registers.
    __device__ __forceinline__ void forget() {
        if constexpr (T::size == 2)
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) asm("" : "+v"(v[j].w[i]));
    }
};

// M sums over a row's threads, the results in all of them.  `red` holds two
// sets of the waves' sums, used in turn, so that one barrier is enough.
template <int G, int M>
__device__ __forceinline__ void row_sums(float (&v)[M], float (*red)[16][M], uint32_t waves, int &turn) {
#pragma unroll
    for (int m = 0; m < M; ++m) v[m] = join_lanes<G ? G : 64, LaneSum>(v[m]);
    if constexpr (G == 0) {
        float(*mine)[M] = red[turn];
        turn ^= 1;
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int m = 0; m < M; ++m) mine[threadIdx.x / 64][m] = v[m];
        __syncthreads();
        const uint32_t i = threadIdx.x % 16;
#pragma unroll
        for (int m = 0; m < M; ++m) v[m] = join_lanes<16, LaneSum>(i < waves ? mine[i][m] : 0.0f);
    }
}

// 1 / sqrt(v), rounded once: the approximation (1 ulp) and a Newton step on it,
// r + r (1 - v r r) / 2, whose difference is taken in two parts, from the
// rounded product v r and from its rounding.  (1 / sqrtf rounds twice and takes
// more instructions.)  Values near and in the subnormal range are scaled.
__device__ __forceinline__ float reciprocal_root(float v) {
    const bool tiny = v < 0x1p-100f;
    if (tiny) v *= 0x1p100f;
    const float r = __builtin_amdgcn_rsqf(v), h = v * r;
    const float e = fmaf(-fmaf(v, r, -h), r, fmaf(-h, r, 1.0f));
    const float s = e == e ? fmaf(0.5f * r, e, r) : r;  // not of zero and infinity
    return tiny ? s * 0x1p50f : s;
}

// G: lanes of a row, 256 / G rows a workgroup; 0: a workgroup a row.
// FAR: reads past the caches, with FULL alone.
template <class T, int G, int NV, bool FULL, bool Q8, bool FAR>
__global__ void __launch_bounds__(G ? kOpThreads : 1024) rmsnorm_kernel(const RmsArgs a) {
    using X = Shaped<T, NV, FULL>;
    constexpr int VE = X::VE, ROWS = G ? kOpThreads / G : 1;
    __shared__ float red[2][16][1];
    int turn = 0;
    const uint32_t H = a.hidden, W = G ? G : a.threads;
    uint32_t t = G ? threadIdx.x % G : threadIdx.x;
    if constexpr (G != 8) __builtin_assume(H >= VE);  // over 8 vectors
    const uint32_t nblk = (H + kBlock - 1) / kBlock;
    const uint64_t step = (uint64_t)gridDim.x * ROWS;
    uint64_t row = (uint64_t)blockIdx.x * ROWS + (G ? threadIdx.x / G : 0);
    X x, res;
    auto load = [&](uint64_t r) {
        x.template load<FAR>(a.x, r, H, W, t);
        if (a.residual) res.template load<FAR>(a.residual, r, H, W, t);
    };
    if (X::ahead && row < a.rows) load(row);
    float w[NV][VE];
    if (X::keep_weights)
#pragma unroll
        for (int j = 0; j < NV; ++j) load_weights(a.weight, a.weight_bf16, (j * W + t) * VE, H, w[j]);
    for (; row < a.rows; row += step) {
        if constexpr (X::anew) t = here(t);
        const uint64_t at = row * H * T::size;
        float h[NV][VE], sum[1] = {0.0f};
        if (!X::ahead) load(row);
        // The next row's reads go out before this one's are waited for, or,
        // where y is not in 8 bits, after: at 8192 x 4096 the other order costs 9 %
        // in 8 bits and 5 % else.
        X now = x, now_res = res;
        if (Q8 && X::ahead && row + step < a.rows) load(row + step);
        now.settle(H, W, t);
        if (a.residual) now_res.settle(H, W, t);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            now.unpack(j, h[j]);
            if (a.residual) {
                float r[VE];
                now_res.unpack(j, r);
#pragma unroll
                for (int i = 0; i < VE; ++i) h[j][i] = T::widen(T::narrow(h[j][i] + r[i]));
            }
        }
        if (!Q8 && X::ahead && row + step < a.rows) load(row + step);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (a.residual_out) X::store((char *)a.residual_out + at, (j * W + t) * VE, H, h[j]);
#pragma unroll
            for (int i = 0; i < VE; ++i) sum[0] += h[j][i] * h[j][i];
        }
        row_sums<G>(sum, red, W / 64, turn);
        if constexpr (X::again) t = here(t);
        const float r = reciprocal_root(sum[0] / (float)H + a.eps);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t e = (j * W + t) * VE;
            if (!X::keep_weights) load_weights(a.weight, a.weight_bf16, e, H, w[j]);
            float y[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) y[i] = h[j][i] * r * w[j][i];
            if constexpr (Q8) {
                // Zeros behind the end, where 0 / 0 may have left a NaN.
#pragma unroll
                for (int i = 0; i < VE; ++i) y[i] = e + i < H ? y[i] : 0.0f;
                const float top = __uint_as_float(join_lanes<(G && G < kBlock / VE ? G : kBlock / VE), LaneUMax>(top_bits(y)));
                float scale, inverse;
                block_scale(top, scale, inverse);
#pragma unroll
                for (int i = 0; i < VE; ++i) y[i] *= inverse;
                Raw<VE> q;
                to_e4m3(y, q);
                store_bytes<true>((char *)a.y + row * H, e, H, q);
                if (e % kBlock == 0 && e < H) a.scale[row * nblk + e / kBlock] = scale;
            } else {
                X::store((char *)a.y + at, e, H, y);
            }
        }
    }
}

// Backward.  Every thread keeps the sums of its columns' weight gradients in
// registers over the rows of a partial sum; the rows of one partial are
// those `blocks` apart.
template <class T, int G, int NV, bool FULL>
__global__ void __launch_bounds__(G ? kOpThreads : 1024) rmsnorm_backward_kernel(const RmsBackArgs a) {
    using X = Shaped<T, NV, FULL>;
    constexpr int VE = X::VE, ROWS = G ? kOpThreads / G : 1;
    __shared__ float red[2][16][2];
    __shared__ float cols[G ? G * VE : 1];
    extern __shared__ float4 grads[];  // lean: a row's, each thread its own
    int turn = 0;
    const uint32_t H = a.hidden, W = G ? G : a.threads;
    uint32_t t = G ? threadIdx.x % G : threadIdx.x;
    if constexpr (G != 8) __builtin_assume(H >= VE);  // over 8 vectors
    const int slot = G ? threadIdx.x / G : 0;
    const uint64_t step = (uint64_t)a.blocks * ROWS;
    X h, g, d;
    auto load = [&](uint64_t r) {
        h.template load<true>(a.h, r, H, W, t);
        g.template load<true>(a.dy, r, H, W, t);
        if (!X::lean && a.dres) d.template load<true>(a.dres, r, H, W, t);
    };
    float w[NV][VE];
    if (X::keep_weights)
#pragma unroll
        for (int j = 0; j < NV; ++j) load_weights(a.weight, a.weight_bf16, (j * W + t) * VE, H, w[j]);
    for (uint32_t part = blockIdx.x; part < a.blocks; part += gridDim.x) {
        float dw[NV][VE] = {};
        if constexpr (X::lean)
#pragma unroll
            for (int j = 0; j < X::N / 4; ++j) grads[j * W + t] = make_float4(0, 0, 0, 0);
        uint64_t row = (uint64_t)part * ROWS + slot;
        if (X::ahead && row < a.rows) load(row);
        for (; row < a.rows; row += step) {
            if constexpr (X::anew) t = here(t);
            if (!X::ahead) load(row);
            X now_h = h, now_g = g, now_d = d;
            if (X::ahead && row + step < a.rows) load(row + step);
            now_h.settle(H, W, t);
            now_g.settle(H, W, t);
            if (!X::lean && a.dres) now_d.settle(H, W, t);
            float sums[2] = {0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float u[VE], y[VE];
                now_h.unpack(j, u);
                now_g.unpack(j, y);
                if (!X::keep_weights) load_weights(a.weight, a.weight_bf16, (j * W + t) * VE, H, w[j]);
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    sums[0] += u[i] * u[i];
                    sums[1] += y[i] * w[j][i] * u[i];
                }
            }
            row_sums<G>(sums, red, W / 64, turn);
            if constexpr (X::again) t = here(t);
            const float r = reciprocal_root(sums[0] / (float)H + a.eps);
            const float c = sums[1] / (float)H * r * r;
            now_h.forget(), now_g.forget();
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float u[VE], y[VE], x[VE] = {};
                now_h.unpack(j, u);
                now_g.unpack(j, y);
                if (X::lean && a.dres)
                    load_some<T, FULL>((const char *)a.dres + row * H * T::size, (j * W + t) * VE, H, x);
                else if (a.dres)
                    now_d.unpack(j, x);
                if (!X::keep_weights) load_weights(a.weight, a.weight_bf16, (j * W + t) * VE, H, w[j]);
#pragma unroll
                for (int i = 0; i < VE; ++i) x[i] += r * (y[i] * w[j][i] - u[i] * c);
                if constexpr (X::lean) {
#pragma unroll
                    for (int i = 0; i < VE; i += 4) {
                        float4 &q = grads[(j * VE + i) / 4 * W + t];
                        float4 v = q;
                        v.x += y[i] * (u[i] * r), v.y += y[i + 1] * (u[i + 1] * r);
                        v.z += y[i + 2] * (u[i + 2] * r), v.w += y[i + 3] * (u[i + 3] * r);
                        q = v;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < VE; ++i) dw[j][i] += y[i] * (u[i] * r);
                }
                X::store((char *)a.dx + row * H * T::size, (j * W + t) * VE, H, x);
            }
        }
        if (!a.partial) continue;
        float *out = a.partial + (uint64_t)part * H;
        bool mine = true;  // the threads that hold the sums
        if constexpr (G > 0) {
            // A wave's rows, then the waves in turn, so that the order is
            // fixed.
            constexpr int WAVES = kOpThreads / 64;
            const int wave = threadIdx.x / 64;
#pragma unroll
            for (int i = 0; i < VE; ++i) dw[0][i] = join_groups<G, LaneSum>(dw[0][i]);
            for (int s = 0; s < WAVES; ++s) {
                if (wave == s && threadIdx.x % 64 < G)
#pragma unroll
                    for (int i = 0; i < VE; ++i) {
                        float &c = cols[i * G + t];
                        c = s ? c + dw[0][i] : dw[0][i];
                        if (s == WAVES - 1) dw[0][i] = c;
                    }
                __syncthreads();
            }
            mine = wave == WAVES - 1 && threadIdx.x % 64 < G;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if constexpr (X::lean)
#pragma unroll
                for (int i = 0; i < VE; i += 4) {
                    const float4 v = grads[(j * VE + i) / 4 * W + t];
                    dw[j][i] = v.x, dw[j][i + 1] = v.y, dw[j][i + 2] = v.z, dw[j][i + 3] = v.w;
                }
            if (mine) store_some<EF32>(out, (j * W + t) * VE, H, dw[j]);
        }
    }
}

// dw[e] = the sum of its partial sums: 32 columns (a cache line of each
// partial) by 32 rows of them.
constexpr uint32_t kGradCols = 32;
__global__ void __launch_bounds__(1024) weight_grad_kernel(const float *partial, uint32_t blocks, uint32_t H,
                                                           float *dw) {
    __shared__ float red[32][kGradCols + 1];
    const uint32_t c = threadIdx.x % kGradCols, g = threadIdx.x / kGradCols;
    for (uint32_t e0 = blockIdx.x * kGradCols; e0 < H; e0 += gridDim.x * kGradCols) {
        const uint32_t e = e0 + c;
        float s = 0.0f;
        if (e < H)
#pragma unroll 8
            for (uint32_t b = g; b < blocks; b += 32) s += partial[(uint64_t)b * H + e];
        red[g][c] = s;
        __syncthreads();
        if (g == 0 && e < H) {
            for (int i = 1; i < 32; ++i) s += red[i][c];
            dw[e] = s;
        }
        __syncthreads();
    }
}

// Threads of a row and vectors of a thread: 8 to 64 lanes of a wave or as few
// waves as hold the row.
struct Shape {
    int W, NV;
    bool full;
};
Shape shape_of(size_t hidden, hoccl_dtype_t dt) {
    const size_t per = dt == HOCCL_BF16 ? kVE<EBF16> : kVE<EF32>, v = (hidden + per - 1) / per;
    Shape s;
    if (v <= 64) {
        s = {v <= 8 ? 8 : v <= 16 ? 16 : v <= 32 ? 32 : 64, 1, false};
    } else {
        int n = 1;
        while (v > (size_t)(1024 * n)) n *= 2;
        s = {(int)((v + 64 * n - 1) / (64 * n)) * 64, n, false};
    }
    s.full = (size_t)s.W * s.NV * per == hidden;
    return s;
}
int group_of(Shape s) { return s.W <= 64 ? kOpThreads : s.W; }  // threads of a workgroup
int rows_of(Shape s) { return group_of(s) / s.W; }

// f(T, G, NV, FULL) of a row's element type and shape.
template <class F>
const void *with_shape(hoccl_dtype_t dt, Shape s, F &&f) {
    auto typed = [&](auto g, auto n) {
        if (s.full) return dt == HOCCL_BF16 ? f(EBF16(), g, n, std::true_type()) : f(EF32(), g, n, std::true_type());
        return dt == HOCCL_BF16 ? f(EBF16(), g, n, std::false_type()) : f(EF32(), g, n, std::false_type());
    };
#define HOCCL_SHAPE(g, n) typed(std::integral_constant<int, g>(), std::integral_constant<int, n>())
    switch (s.W) {
    case 8: return HOCCL_SHAPE(8, 1);
    case 16: return HOCCL_SHAPE(16, 1);
    case 32: return HOCCL_SHAPE(32, 1);
    case 64: return HOCCL_SHAPE(64, 1);
    }
    switch (s.NV) {
    case 1: return HOCCL_SHAPE(0, 1);
    case 2: return HOCCL_SHAPE(0, 2);
    case 4: return HOCCL_SHAPE(0, 4);
    }
#undef HOCCL_SHAPE
    // fp32 alone: 32768 bf16 are four vectors a thread.
    return f(EF32(), std::integral_constant<int, 0>(), std::integral_constant<int, 8>(), std::false_type());
}

}  // namespace

// Calls of more bytes read past the caches: half of what the last of them (256
// MiB) holds.  Rows of whole vectors, us with plain reads / past the caches,
// where a call finds its inputs: nowhere (many tensors in turn), in what three
// calls in turn leave, or all of them (the same tensors again):
//
//   bf16 with a residual   64 MB  14.5 / 13.1   10.9 / 13.1    9.3 / 12.4
//                         128     25.4 / 23.5   22.5 / 22.7   20.1 / 22.7
//                         160     31.2 / 27.4   31.0 / 26.8   24.8 / 26.9
//                         260     49.9 / 42.4   50.7 / 43.5   41.6 / 44.5
//   fp32                   64     14.6 / 13.9   11.0 / 13.0   10.9 / 12.8
//                         128     25.3 / 24.5   25.4 / 23.1   20.6 / 23.6
//                         256     49.6 / 49.1   47.8 / 46.9   39.0 / 41.5
//   y in 8 bits            59     13.3 / 13.0   11.8 / 13.1   10.0 / 12.5
//                         160     30.8 / 29.6   29.5 / 29.4   27.9 / 29.0
//                         256     49.5 / 47.7   48.7 / 46.2   41.6 / 47.2
//
// The middle one, a step's calls one after another, crosses at about 128 MB, for
// y in 8 bits at 160.
constexpr unsigned long long kFarBytes = 128ull << 20;

// Threads of a CU's workgroups in the forward pass: what it holds.  A quarter
// of them: 8 % longer at 8192 x 4096, 12 % at 4096 x 2048 into 8 bits.
constexpr unsigned kForwardThreads = 2048;
// Workgroups of the backward pass, and partial sums: as many for each of 256
// CUs as make about 512 threads.  16384 x 4096 takes 8 % longer with 1024
// threads; but rows under 512 threads whose last vectors are not whole leave
// lanes idle and wait more (640 bf16: 24 % less with 1024; 5003, 640 threads, 5
// % more).
size_t backward_groups(Shape s) {
    const int threads = group_of(s), most = s.full || threads >= 512 ? 512 : 1024;
    return 256 * (size_t)std::max(1, (most + threads / 2) / threads);
}

unsigned long long rmsnorm_workgroups(size_t rows, size_t hidden, hoccl_dtype_t dt, int cus) {
    const Shape s = shape_of(hidden, dt);
    const unsigned long long groups = (rows + rows_of(s) - 1) / rows_of(s);
    return std::min(groups, (unsigned long long)kForwardThreads / group_of(s) * cus);
}

hipError_t launch_rmsnorm(RmsArgs a, hoccl_dtype_t dt, unsigned long long bytes, int wg, hipStream_t s) {
    const bool far = bytes > kFarBytes;  // with FULL alone
    const Shape sh = shape_of(a.hidden, dt);
    const void *k = with_shape(dt, sh, [&](auto type, auto g, auto n, auto full) -> const void * {
        using T = decltype(type);
        constexpr int G = decltype(g)::value, NV = decltype(n)::value;
        constexpr bool FULL = decltype(full)::value;
        if (a.scale)
            return far ? (const void *)rmsnorm_kernel<T, G, NV, FULL, true, FULL>
                       : (const void *)rmsnorm_kernel<T, G, NV, FULL, true, false>;
        return far ? (const void *)rmsnorm_kernel<T, G, NV, FULL, false, FULL>
                   : (const void *)rmsnorm_kernel<T, G, NV, FULL, false, false>;
    });
    a.threads = (uint32_t)sh.W;
    void *args[] = {(void *)&a};
    return hipLaunchKernel(k, dim3((unsigned)wg), dim3(group_of(sh)), args, 0, s);
}

uint32_t rmsnorm_backward_blocks(size_t rows, size_t hidden, hoccl_dtype_t dt) {
    const Shape s = shape_of(hidden, dt);
    const size_t groups = (rows + rows_of(s) - 1) / rows_of(s);
    return (uint32_t)std::min(groups, backward_groups(s));
}

hipError_t launch_rmsnorm_backward(RmsBackArgs a, hoccl_dtype_t dt, int wg, hipStream_t s) {
    const Shape sh = shape_of(a.hidden, dt);
    size_t lds = 0;
    const void *k = with_shape(dt, sh, [&](auto type, auto g, auto n, auto full) -> const void * {
        using T = decltype(type);
        constexpr int G = decltype(g)::value, NV = decltype(n)::value;
        constexpr bool FULL = decltype(full)::value;
        using X = Shaped<T, NV, FULL>;
        if (X::lean) lds = (size_t)sh.W * X::N * 4;
        return (const void *)rmsnorm_backward_kernel<T, G, NV, FULL>;
    });
    if (lds > (size_t)48 << 10) {  // up to 128 KiB of a CU's 160
        const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    a.threads = (uint32_t)sh.W;
    void *args[] = {(void *)&a};
    return hipLaunchKernel(k, dim3((unsigned)wg), dim3(group_of(sh)), args, lds, s);
}

uint32_t rmsnorm_grad_workgroups(size_t hidden) { return (uint32_t)((hidden + kGradCols - 1) / kGradCols); }

hipError_t launch_rmsnorm_weight_grad(const float *partial, uint32_t blocks, uint32_t hidden, float *dweight, int wg,
                                      hipStream_t s) {
    void *args[] = {(void *)&partial, (void *)&blocks, (void *)&hidden, (void *)&dweight};
    return hipLaunchKernel((const void *)weight_grad_kernel, dim3((unsigned)wg), dim3(1024), args, 0, s);
}

}  // namespace hoccl
