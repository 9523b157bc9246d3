// Device helpers of the operators' kernels (adamw.hip, rmsnorm.hip,
// balance.hip): vectors of elements at any element address, bf16 and e4m3
// conversions, and sums and maxima over neighbouring lanes.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace hoccl {

// The compute units take 4-, 8- and 16-byte global accesses at any byte
// address, so the same instructions serve aligned and misaligned tensors.
typedef uint32_t v4u __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t v2u __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t v1u __attribute__((aligned(1)));

template <int BYTES>
struct Raw {
    uint32_t w[BYTES / 4];
};

template <bool NT = false, int BYTES>
__device__ __forceinline__ void load_raw(Raw<BYTES> &r, const void *p) {
    if constexpr (BYTES == 4) {
        r.w[0] = NT ? __builtin_nontemporal_load((const v1u *)p) : *(const v1u *)p;
    } else if constexpr (BYTES == 8) {
        const v2u v = NT ? __builtin_nontemporal_load((const v2u *)p) : *(const v2u *)p;
        r.w[0] = v.x, r.w[1] = v.y;
    } else {
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) {
            const v4u v = NT ? __builtin_nontemporal_load((const v4u *)p + i) : ((const v4u *)p)[i];
            r.w[4 * i] = v.x, r.w[4 * i + 1] = v.y, r.w[4 * i + 2] = v.z, r.w[4 * i + 3] = v.w;
        }
    }
}
template <bool NT = false, int BYTES>
__device__ __forceinline__ void store_raw(void *p, const Raw<BYTES> &r) {
    if constexpr (BYTES == 4) {
        if (NT)
            __builtin_nontemporal_store(r.w[0], (v1u *)p);
        else
            *(v1u *)p = r.w[0];
    } else if constexpr (BYTES == 8) {
        const v2u v = {r.w[0], r.w[1]};
        if (NT)
            __builtin_nontemporal_store(v, (v2u *)p);
        else
            *(v2u *)p = v;
    } else {
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) {
            const v4u v = {r.w[4 * i], r.w[4 * i + 1], r.w[4 * i + 2], r.w[4 * i + 3]};
            if (NT)
                __builtin_nontemporal_store(v, (v4u *)p + i);
            else
                ((v4u *)p)[i] = v;
        }
    }
}

// Element types: N elements in a Raw, to and from floats.
struct EF32 {
    using S = float;
    static constexpr int size = 4;
    static __device__ __forceinline__ float widen(float v) { return v; }
    static __device__ __forceinline__ float narrow(float f) { return f; }
    template <int N>
    static __device__ __forceinline__ void unpack(const Raw<4 * N> &r, float (&f)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = __uint_as_float(r.w[i]);
    }
    template <int N>
    static __device__ __forceinline__ void pack(const float (&f)[N], Raw<4 * N> &r) {
#pragma unroll
        for (int i = 0; i < N; ++i) r.w[i] = __float_as_uint(f[i]);
    }
};
struct EBF16 {
    using S = uint16_t;
    static constexpr int size = 2;
    static __device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
    // Round to nearest even; NaN stays NaN.
    static __device__ __forceinline__ uint16_t narrow(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
    template <int N>
    static __device__ __forceinline__ void unpack(const Raw<2 * N> &r, float (&f)[N]) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            f[2 * i] = __uint_as_float(r.w[i] << 16);
            f[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
        }
    }
    template <int N>
    static __device__ __forceinline__ void pack(const float (&f)[N], Raw<2 * N> &r) {
        typedef float f2 __attribute__((ext_vector_type(2)));
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {  // one instruction converts and packs two
            const f2 x = {f[2 * i], f[2 * i + 1]};
            r.w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, b2));
        }
    }
};

// The same value, which the compiler takes for another.  The element-by-element
// ends below start with it, so that their comparisons stay there: hoisted out
// of the callers' loops they took a dozen registers and as many instructions
// of every pass.
template <typename V>
__device__ __forceinline__ V here(V v) {
    asm volatile("" : "+v"(v));
    return v;
}

// r shifted down by `bytes` (0 to B), zeros from above.
template <int B>
__device__ __forceinline__ void shift_down(Raw<B> &r, uint32_t bytes) {
    constexpr int W = B / 4;
#pragma unroll
    for (int s = W; s >= 1; s /= 2)
        if (bytes & (4 * s))
#pragma unroll
            for (int i = 0; i < W; ++i) r.w[i] = i + s < W ? r.w[i + s] : 0;
#pragma unroll
    for (int i = 0; i < W; ++i)
        r.w[i] = __builtin_amdgcn_alignbit(i + 1 < W ? r.w[i + 1] : 0, r.w[i], bytes % 4 * 8);
}

// N elements of `p` from element e on, in two steps.  load_window reads them
// or, where fewer than N are left before `end`, the N that end there, so that
// every lane makes the same one read; settle_window moves what was read to
// its place and makes zeros of elements at and behind `end`.  (Read element by
// element, the ends of rows of 5003 bf16 waited for memory eight times: their
// gradients took 1.6 times as long.)  Only where there are fewer than N
// elements in all are they read one by one.  Any e is allowed.
template <class T, bool NT = false, int B, typename I>
__device__ __forceinline__ void load_window(const void *p, I e, I end, Raw<B> &r) {
    constexpr I N = B / T::size;
    if (end >= N) {
        load_raw<NT>(r, (const char *)p + (size_t)(e + N <= end ? e : end - N) * T::size);
    } else {
        e = here(e);
#pragma unroll
        for (int i = 0; i < B / 4; ++i) r.w[i] = 0;
#pragma unroll
        for (int i = 0; i < (int)N; ++i)
            if (e + i < end) {
                if constexpr (T::size == 4) r.w[i] = ((const uint32_t *)p)[e + i];
                else if constexpr (T::size == 2) r.w[i / 2] |= (uint32_t)((const uint16_t *)p)[e + i] << (16 * (i % 2));
                else r.w[i / 4] |= (uint32_t)((const uint8_t *)p)[e + i] << (8 * (i % 4));
            }
    }
}
template <class T, int B, typename I>
__device__ __forceinline__ void settle_window(I e, I end, Raw<B> &r) {
    constexpr I N = B / T::size;
    if (end >= N && e + N > end) {
        const I s = e + N - end;
        shift_down(r, (uint32_t)(s < N ? s : N) * T::size);
    }
}

// Both steps: N elements, as numbers.
template <class T, bool NT = false, int N, typename I>
__device__ __forceinline__ void load_some(const void *p, I e, I end, float (&f)[N]) {
    Raw<T::size * N> r;
    load_window<T, NT>(p, e, end, r);
    settle_window<T>(e, end, r);
    T::template unpack<N>(r, f);
}
// Writes those of the N elements that lie before `end`.
template <class T, bool NT = false, int N, typename I>
__device__ __forceinline__ void store_some(void *p, I e, I end, const float (&f)[N]) {
    if (e + N <= end) {
        Raw<T::size * N> r;
        T::template pack<N>(f, r);
        store_raw<NT>((char *)p + e * T::size, r);
    } else {
        e = here(e);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (e + i < end) ((typename T::S *)p)[e + i] = T::narrow(f[i]);
    }
}

// ---- lanes -------------------------------------------------------------------

struct LaneSum {
    template <typename V>
    static __device__ __forceinline__ V join(V a, V b) { return a + b; }
};
struct LaneMax {  // NaN gives way to a number
    static __device__ __forceinline__ float join(float a, float b) { return fmaxf(a, b); }
};
struct LaneUMax {
    static __device__ __forceinline__ uint32_t join(uint32_t a, uint32_t b) { return a > b ? a : b; }
};
struct LaneOr {
    static __device__ __forceinline__ uint32_t join(uint32_t a, uint32_t b) { return a | b; }
};

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __uint_as_float(dpp<CTRL>(__float_as_uint(v)));
}
template <int CTRL>
__device__ __forceinline__ int dpp(int v) {
    return (int)dpp<CTRL>((uint32_t)v);
}
struct U2 {
    uint32_t a, b;
};
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
    const U2 x = __builtin_bit_cast(U2, v);
    return __builtin_bit_cast(double, U2{dpp<CTRL>(x.a), dpp<CTRL>(x.b)});
}

// v of the other row of 16 (SWAP32: of the other half of the wave) joined
// with the lane's own.
template <bool SWAP32>
__device__ __forceinline__ U2 swap_rows(uint32_t v) {
    if constexpr (SWAP32) {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return {r[0], r[1]};
    } else {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return {r[0], r[1]};
    }
}
template <bool SWAP32, class J, typename V>
__device__ __forceinline__ V join_rows(V v) {
    if constexpr (sizeof(V) == 8) {
        const U2 x = __builtin_bit_cast(U2, v), lo = swap_rows<SWAP32>(x.a), hi = swap_rows<SWAP32>(x.b);
        return J::join(__builtin_bit_cast(V, U2{lo.a, hi.a}), __builtin_bit_cast(V, U2{lo.b, hi.b}));
    } else {
        const U2 r = swap_rows<SWAP32>(__builtin_bit_cast(uint32_t, v));
        return J::join(__builtin_bit_cast(V, r.a), __builtin_bit_cast(V, r.b));
    }
}

// v of every lane joined over each aligned group of L lanes (a power of two
// up to 64), the result in all of them.  A group's lanes take part together;
// other groups need not.  Groups
// of up to 16 exchange by DPP: neighbours, pairs, then the mirrored half row
// and the mirrored row (a group's lanes hold the same value by then, so that
// a mirror is as good as an exchange); rows by the swaps of rows.
template <int L, class J, typename V>
__device__ __forceinline__ V join_lanes(V v) {
    if constexpr (L >= 2) v = J::join(v, dpp<0xB1>(v));    // quad_perm 1,0,3,2
    if constexpr (L >= 4) v = J::join(v, dpp<0x4E>(v));    // quad_perm 2,3,0,1
    if constexpr (L >= 8) v = J::join(v, dpp<0x141>(v));   // row_half_mirror
    if constexpr (L >= 16) v = J::join(v, dpp<0x140>(v));  // row_mirror
    if constexpr (L >= 32) v = join_rows<false, J>(v);
    if constexpr (L >= 64) v = join_rows<true, J>(v);
    return v;
}

// The other way round: v joined over the wave's lanes that have the same place
// in their groups of L.  For whole waves.
template <int L, class J, typename V>
__device__ __forceinline__ V join_groups(V v) {
#pragma unroll
    for (int o = L; o < 8; o *= 2) v = J::join(v, (V)__shfl_xor(v, o));
    if constexpr (L <= 8) v = J::join(v, dpp<0x128>(v));  // row_ror:8
    if constexpr (L <= 16) v = join_rows<false, J>(v);
    if constexpr (L <= 32) v = join_rows<true, J>(v);
    return v;
}

// ---- 8 bits: e4m3 with one fp32 scale for each block of 128 elements ------------

constexpr int kBlock = 128;
constexpr float kTop = 448.0f;                  // the largest e4m3 value
constexpr float kTiny = 7.888609052210118e-31f;  // 2^-100: blocks that hold less are held as zeros
constexpr float kLeast = 0.001953125f;           // 2^-9, the smallest e4m3 value above zero

// The scale of a block and what its elements are multiplied by.  `top` is
// the block's largest magnitude; where that is infinite or NaN the whole
// block reads back as NaN.
__device__ __forceinline__ void block_scale(float top, float &scale, float &inverse) {
    const bool some = !(top < kTiny);
    scale = some ? top / kTop : 0.0f;
    inverse = some ? kTop / top : 0.0f;
}

// Largest magnitude of N values, as its bits: compared as integers, so that
// an infinity or a NaN wins.
template <int N>
__device__ __forceinline__ uint32_t top_bits(const float (&f)[N]) {
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) t = LaneUMax::join(t, __float_as_uint(f[i]) & 0x7fffffffu);
    return t;
}

struct EByte {  // windows of e4m3 bytes
    static constexpr int size = 1;
};

// N (4 or 8) floats of magnitude up to 448 to e4m3 bytes (round to nearest
// even) and back.
template <int N>
__device__ __forceinline__ void to_e4m3(const float (&f)[N], Raw<N> &r) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false);
        r.w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], w, true);
    }
}
template <int N>
__device__ __forceinline__ void from_e4m3(const Raw<N> &r, float (&f)[N]) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.w[i], false);
        const auto b = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.w[i], true);
        f[4 * i] = a[0], f[4 * i + 1] = a[1], f[4 * i + 2] = b[0], f[4 * i + 3] = b[1];
    }
}
template <bool NT = false, int N, typename I>
__device__ __forceinline__ void store_bytes(void *p, I e, I end, const Raw<N> &r) {
    if (e + N <= end) {
        store_raw<NT>((char *)p + e, r);
    } else {
        e = here(e);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (e + i < end) ((uint8_t *)p)[e + i] = (uint8_t)(r.w[i / 4] >> (8 * (i % 4)));
    }
}

template <typename A>
__device__ __forceinline__ const A &kernel_args() {
    return *(const A *)__builtin_amdgcn_kernarg_segment_ptr();
}

}  // namespace hoccl
