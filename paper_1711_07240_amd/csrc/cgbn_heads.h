// Pieces of a head's row as a lane holds them: what the head norm and the rotation have in common.
#pragma once

#include "cgbn_kernels.h"

namespace cgbn {
namespace {

// N neighbouring floats at any float's address
template <int N> __device__ __forceinline__ void load_floats(const float* p, float (&v)[N])
{
    typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            const f32x4_any t = *reinterpret_cast<const f32x4_any*>(p + k);
            v[k] = t.x; v[k + 1] = t.y; v[k + 2] = t.z; v[k + 3] = t.w;
        }
    } else if constexpr (N == 1) {
        v[0] = *p;
    } else {
        static_assert(N == 2, "");
        typedef float f32x2_any __attribute__((ext_vector_type(2), aligned(4)));
        const f32x2_any t = *reinterpret_cast<const f32x2_any*>(p);
        v[0] = t.x; v[1] = t.y;
    }
}

// E values as they are stored: 16 bytes, or fewer where rows or halves do not go in those
template <typename T, int E> struct Chunk {
    static_assert(E * sizeof(T) == 16, "");
    typedef typename Elem<T>::Raw Raw;
    static __device__ __forceinline__ Raw load(const T* p) { return Elem<T>::load_raw(p); }
    static __device__ __forceinline__ void unpack(const Raw& v, float (&f)[E]) { Elem<T>::unpack(v, f); }
    template <bool NT> static __device__ __forceinline__ void store(T* p, const float (&f)[E])
    {
        u32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (E == 8) v[k] = f32x2_to_bf16x2(f[2 * k], f[2 * k + 1]);
            else v[k] = __float_as_uint(f[k]);
        }
        if constexpr (NT) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
        else *reinterpret_cast<u32x4*>(p) = v;
    }
};
template <> struct Chunk<bf16_t, 4> {
    typedef uint2 Raw;
    static __device__ __forceinline__ Raw load(const bf16_t* p) { return *reinterpret_cast<const uint2*>(p); }
    static __device__ __forceinline__ void unpack(const Raw& v, float (&f)[4])
    {
        f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
        f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
    }
    template <bool NT> static __device__ __forceinline__ void store(bf16_t* p, const float (&f)[4])
    {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        const u32x2 v = {f32x2_to_bf16x2(f[0], f[1]), f32x2_to_bf16x2(f[2], f[3])};
        if constexpr (NT) __builtin_nontemporal_store(v, reinterpret_cast<u32x2*>(p));
        else *reinterpret_cast<u32x2*>(p) = v;
    }
};

template <> struct Chunk<bf16_t, 2> {
    typedef uint32_t Raw;
    static __device__ __forceinline__ Raw load(const bf16_t* p) { return *reinterpret_cast<const uint32_t*>(p); }
    static __device__ __forceinline__ void unpack(const Raw& v, float (&f)[2])
    {
        f[0] = __uint_as_float(v << 16);
        f[1] = __uint_as_float(v & 0xffff0000u);
    }
    template <bool> static __device__ __forceinline__ void store(bf16_t* p, const float (&f)[2])
    {
        *reinterpret_cast<uint32_t*>(p) = f32x2_to_bf16x2(f[0], f[1]);
    }
};
template <> struct Chunk<float, 2> {
    typedef float2 Raw;
    static __device__ __forceinline__ Raw load(const float* p) { return *reinterpret_cast<const float2*>(p); }
    static __device__ __forceinline__ void unpack(const Raw& v, float (&f)[2]) { f[0] = v.x; f[1] = v.y; }
    template <bool> static __device__ __forceinline__ void store(float* p, const float (&f)[2]) { *reinterpret_cast<float2*>(p) = make_float2(f[0], f[1]); }
};
// (bits, as a 32-bit register holds them: a value that is converted where it is loaded, or kept in 16, is waited for there: 80 heads of 39,
// 15994 tokens, backward 553 and 269 us, and so 170)
template <> struct Chunk<bf16_t, 1> {
    typedef uint32_t Raw;
    static __device__ __forceinline__ Raw load(const bf16_t* p) { return p->bits; }
    static __device__ __forceinline__ void unpack(const Raw& v, float (&f)[1]) { f[0] = __uint_as_float(v << 16); }
    template <bool> static __device__ __forceinline__ void store(bf16_t* p, const float (&f)[1]) { Elem<bf16_t>::store1(p, f[0]); }
};
template <> struct Chunk<float, 1> {
    typedef float Raw;
    static __device__ __forceinline__ Raw load(const float* p) { return *p; }
    static __device__ __forceinline__ void unpack(const Raw& v, float (&f)[1]) { f[0] = v; }
    template <bool> static __device__ __forceinline__ void store(float* p, const float (&f)[1]) { *p = f[0]; }
};

template <typename T, int E> __device__ __forceinline__ typename Chunk<T, E>::Raw load_chunk(const T* row, int c)
{
    typename Chunk<T, E>::Raw v{};
    if (c >= 0) v = Chunk<T, E>::load(row + c);
    return v;
}

}  // namespace
}  // namespace cgbn
