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
// One pass over the data: W threads hold a whole row in registers (up to NV
// vectors of 16 bytes each), so that what is read is read once.  Rows of up
// to four vectors a lane take one wave, with no exchange through LDS; longer
// ones a workgroup of 256 or 1024.  Sums are in fp32, in an order that goes
// by the row's length alone.
//
// Bound by memory: 8 bytes an element (bf16 with a residual), 7 with y in 8
// bits; backward 8 bytes and the partial sums of the weight's gradient.
#include <type_traits>

#include "lanes.h"
#include "shard_ops.h"

namespace hoccl {
namespace {

template <class T>
constexpr int kVE = 16 / T::size;  // elements of a vector

__device__ __forceinline__ float load_weight(const void *w, int bf16, uint32_t e) {
    return bf16 ? EBF16::widen(((const uint16_t *)w)[e]) : ((const float *)w)[e];
}

// Sum over the W threads of a row, the result in all of them.  `red` holds
// two sets of W / 64 sums, used in turn, so that one barrier a sum is enough.
template <int W>
__device__ __forceinline__ float row_sum(float v, float (*red)[16], int &turn) {
    v = join_lanes<64, LaneSum>(v);
    if constexpr (W > 64) {
        float *mine = red[turn];
        turn ^= 1;
        if (threadIdx.x % 64 == 0) mine[threadIdx.x / 64] = v;
        __syncthreads();
        v = mine[0];
#pragma unroll
        for (int i = 1; i < W / 64; ++i) v += mine[i];
    }
    return v;
}

template <class T, int W, int NV, bool Q8>
__global__ void __launch_bounds__(W < kOpThreads ? kOpThreads : W) rmsnorm_kernel(const RmsArgs a) {
    constexpr int VE = kVE<T>;
    constexpr int ROWS = W < kOpThreads ? kOpThreads / W : 1;  // rows of a workgroup
    __shared__ float red[2][16];
    int turn = 0;
    const uint32_t H = a.hidden, t = threadIdx.x % W, nblk = (H + kBlock - 1) / kBlock;
    float w[NV][VE];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            const uint32_t e = (j * W + t) * VE + i;
            w[j][i] = e < H ? load_weight(a.weight, a.weight_bf16, e) : 0.0f;
        }
    for (uint64_t row = (uint64_t)blockIdx.x * ROWS + threadIdx.x / W; row < a.rows; row += (uint64_t)gridDim.x * ROWS) {
        const uint64_t at = row * H * T::size;
        float h[NV][VE], sum = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) load_some<T>((const char *)a.x + at, (j * W + t) * VE, H, h[j]);
        if (a.residual) {
            float r[NV][VE];
#pragma unroll
            for (int j = 0; j < NV; ++j) load_some<T>((const char *)a.residual + at, (j * W + t) * VE, H, r[j]);
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VE; ++i) h[j][i] = T::widen(T::narrow(h[j][i] + r[j][i]));
        }
        if (a.residual_out) {
#pragma unroll
            for (int j = 0; j < NV; ++j) store_some<T>((char *)a.residual_out + at, (j * W + t) * VE, H, h[j]);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VE; ++i) sum += h[j][i] * h[j][i];
        sum = row_sum<W>(sum, red, turn);
        const float r = 1.0f / __builtin_sqrtf(sum / (float)H + a.eps);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t e = (j * W + t) * VE;
            float y[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) y[i] = h[j][i] * r * w[j][i];
            if constexpr (Q8) {
                // Zeros behind the end, where 0 / 0 may have left a NaN.
#pragma unroll
                for (int i = 0; i < VE; ++i) y[i] = e + i < H ? y[i] : 0.0f;
                const float top = __uint_as_float(join_lanes<kBlock / VE, LaneUMax>(top_bits(y)));
                float scale, inverse;
                block_scale(top, scale, inverse);
#pragma unroll
                for (int i = 0; i < VE; ++i) y[i] *= inverse;
                Raw<VE> q;
                to_e4m3(y, q);
                store_bytes((char *)a.y + row * H, e, H, q);
                if (e % kBlock == 0 && e < H) a.scale[row * nblk + e / kBlock] = scale;
            } else {
                store_some<T>((char *)a.y + at, e, H, y);
            }
        }
    }
}

// Backward.  Every thread keeps the sums of its columns' weight gradients in
// registers over the rows of a partial sum; the rows of one partial are
// those `blocks` apart.
template <class T, int W, int NV>
__global__ void __launch_bounds__(W < kOpThreads ? kOpThreads : W) rmsnorm_backward_kernel(const RmsBackArgs a) {
    constexpr int VE = kVE<T>;
    constexpr int ROWS = W < kOpThreads ? kOpThreads / W : 1;
    __shared__ float red[2][16];
    __shared__ float cols[ROWS > 1 ? W * NV * VE : 1];
    int turn = 0;
    const uint32_t H = a.hidden, t = threadIdx.x % W, slot = threadIdx.x / W;
    float w[NV][VE];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            const uint32_t e = (j * W + t) * VE + i;
            w[j][i] = e < H ? load_weight(a.weight, a.weight_bf16, e) : 0.0f;
        }
    for (uint32_t part = blockIdx.x; part < a.blocks; part += gridDim.x) {
        float dw[NV][VE] = {};
        for (uint64_t row = (uint64_t)part * ROWS + slot; row < a.rows; row += (uint64_t)a.blocks * ROWS) {
            const uint64_t at = row * H * T::size;
            float h[NV][VE], g[NV][VE], d[NV][VE], sum = 0.0f, dot = 0.0f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const uint32_t e = (j * W + t) * VE;
                load_some<T>((const char *)a.h + at, e, H, h[j]);
                load_some<T>((const char *)a.dy + at, e, H, g[j]);
            }
            if (a.dres) {
#pragma unroll
                for (int j = 0; j < NV; ++j) load_some<T>((const char *)a.dres + at, (j * W + t) * VE, H, d[j]);
            }
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    sum += h[j][i] * h[j][i];
                    dot += g[j][i] * w[j][i] * h[j][i];
                }
            sum = row_sum<W>(sum, red, turn);
            dot = row_sum<W>(dot, red, turn);
            const float r = 1.0f / __builtin_sqrtf(sum / (float)H + a.eps);
            const float c = dot / (float)H * r * r;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float x[VE];
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    x[i] = r * (g[j][i] * w[j][i] - h[j][i] * c);
                    if (a.dres) x[i] += d[j][i];
                    dw[j][i] += g[j][i] * (h[j][i] * r);
                }
                store_some<T>((char *)a.dx + at, (j * W + t) * VE, H, x);
            }
        }
        if (!a.partial) continue;
        float *out = a.partial + (uint64_t)part * H;
        if constexpr (ROWS > 1) {
            // The workgroup's rows in turn, so that the order is fixed.
            for (int s = 0; s < ROWS; ++s) {
                if ((int)slot == s)
#pragma unroll
                    for (int j = 0; j < NV; ++j)
#pragma unroll
                        for (int i = 0; i < VE; ++i) {
                            float &c = cols[(j * VE + i) * W + t];
                            c = s ? c + dw[j][i] : dw[j][i];
                            if (s == ROWS - 1) dw[j][i] = c;
                        }
                __syncthreads();
            }
            if (slot != ROWS - 1) continue;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) store_some<EF32>(out, (j * W + t) * VE, H, dw[j]);
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

// Threads of a row and vectors of a thread.
struct Shape {
    int W, NV;
};
Shape shape_of(size_t hidden, hoccl_dtype_t dt) {
    const size_t v = (hidden + 16 / (dt == HOCCL_BF16 ? 2 : 4) - 1) / (16 / (dt == HOCCL_BF16 ? 2 : 4));
    auto nv = [&](size_t w) { return v <= w ? 1 : v <= 2 * w ? 2 : v <= 4 * w ? 4 : 8; };
    if (v <= 256) return {64, nv(64)};
    if (v <= 1024) return {256, nv(256)};
    return {1024, nv(1024)};
}
int rows_of(int W) { return W < kOpThreads ? kOpThreads / W : 1; }

// f(T, W, NV) of a row's element type and shape.
template <class F>
const void *with_shape(hoccl_dtype_t dt, Shape s, F &&f) {
#define HOCCL_SHAPE(w, n)                                                                  \
    if (s.W == w && s.NV == n)                                                             \
        return dt == HOCCL_BF16                                                            \
                   ? f(EBF16(), std::integral_constant<int, w>(), std::integral_constant<int, n>()) \
                   : f(EF32(), std::integral_constant<int, w>(), std::integral_constant<int, n>())
    HOCCL_SHAPE(64, 1);
    HOCCL_SHAPE(64, 2);
    HOCCL_SHAPE(64, 4);
    HOCCL_SHAPE(256, 2);
    HOCCL_SHAPE(256, 4);
    HOCCL_SHAPE(1024, 2);
    HOCCL_SHAPE(1024, 4);
#undef HOCCL_SHAPE
    // fp32 alone: 32768 bf16 are four vectors a thread.
    return f(EF32(), std::integral_constant<int, 1024>(), std::integral_constant<int, 8>());
}

}  // namespace

unsigned long long rmsnorm_workgroups(size_t rows, size_t hidden, hoccl_dtype_t dt, int cus) {
    const Shape s = shape_of(hidden, dt);
    const unsigned long long groups = (rows + rows_of(s.W) - 1) / rows_of(s.W);
    return groups < 8ull * cus ? groups : 8ull * cus;
}

hipError_t launch_rmsnorm(const RmsArgs &a, hoccl_dtype_t dt, int wg, hipStream_t s) {
    const Shape sh = shape_of(a.hidden, dt);
    const void *k = with_shape(dt, sh, [&](auto type, auto w, auto n) -> const void * {
        using T = decltype(type);
        constexpr int W = decltype(w)::value, NV = decltype(n)::value;
        return a.scale ? (const void *)rmsnorm_kernel<T, W, NV, true> : (const void *)rmsnorm_kernel<T, W, NV, false>;
    });
    void *args[] = {(void *)&a};
    return hipLaunchKernel(k, dim3((unsigned)wg), dim3(sh.W < kOpThreads ? kOpThreads : sh.W), args, 0, s);
}

uint32_t rmsnorm_backward_blocks(size_t rows, size_t hidden, hoccl_dtype_t dt) {
    const size_t per = (size_t)rows_of(shape_of(hidden, dt).W), groups = (rows + per - 1) / per;
    return (uint32_t)(groups < 1024 ? groups : 1024);
}

hipError_t launch_rmsnorm_backward(const RmsBackArgs &a, hoccl_dtype_t dt, int wg, hipStream_t s) {
    const Shape sh = shape_of(a.hidden, dt);
    const void *k = with_shape(dt, sh, [&](auto type, auto w, auto n) -> const void * {
        return (const void *)rmsnorm_backward_kernel<decltype(type), decltype(w)::value, decltype(n)::value>;
    });
    void *args[] = {(void *)&a};
    return hipLaunchKernel(k, dim3((unsigned)wg), dim3(sh.W < kOpThreads ? kOpThreads : sh.W), args, 0, s);
}

uint32_t rmsnorm_grad_workgroups(size_t hidden) { return (uint32_t)((hidden + kGradCols - 1) / kGradCols); }

hipError_t launch_rmsnorm_weight_grad(const float *partial, uint32_t blocks, uint32_t hidden, float *dweight, int wg,
                                      hipStream_t s) {
    void *args[] = {(void *)&partial, (void *)&blocks, (void *)&hidden, (void *)&dweight};
    return hipLaunchKernel((const void *)weight_grad_kernel, dim3((unsigned)wg), dim3(1024), args, 0, s);
}

}  // namespace hoccl
