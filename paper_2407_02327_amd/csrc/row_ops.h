// What the row-wise kernels (layer norm, logits) share: rows of fp32, binary16 or bfloat16 read and written in 16-byte vectors at
// any element alignment, and reductions over 16 and 64 lanes on the data-parallel primitives.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace qsync {

namespace {

typedef unsigned row_v4u32 __attribute__((ext_vector_type(4)));
// A row of an odd number of 16-bit elements starts at any even address.  Global memory takes 16-byte accesses at any address here, so
// one form serves every leading dimension (layer norm of 2187 x 1001 fp32 6.3 us, 2187 x 1024 6.0).
typedef row_v4u32 row_v4u32_a2 __attribute__((aligned(2)));
typedef row_v4u32 row_v4u32_a4 __attribute__((aligned(4)));

template <typename T> struct RowType;
template <> struct RowType<float>
{
    static constexpr int      N = 4, kCode = kF32;      // elements of a 16-byte vector
    static constexpr uint32_t kMinusInf = 0xFF800000u;  // vector words of absent logits
    typedef row_v4u32_a4 vec_t;
    template <int E> __device__ static __forceinline__ float get(const row_v4u32& w) { return __uint_as_float(w[E]); }
    __device__ static __forceinline__ row_v4u32 pack(const float (&v)[4])
    {
        return row_v4u32{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
};
template <> struct RowType<_Float16>
{
    static constexpr int      N = 8, kCode = kF16;
    static constexpr uint32_t kMinusInf = 0xFC00FC00u;
    typedef row_v4u32_a2 vec_t;
    template <int E> __device__ static __forceinline__ float get(const row_v4u32& w)
    {
        return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(E % 2 ? w[E / 2] >> 16 : w[E / 2])));
    }
    __device__ static __forceinline__ row_v4u32 pack(const float (&v)[8])      // to nearest even
    {
        row_v4u32 w;
#pragma unroll
        for(int i = 0; i < 4; ++i)
            w[i] = static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<_Float16>(v[2 * i])))
                   | static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<_Float16>(v[2 * i + 1]))) << 16;
        return w;
    }
};
template <> struct RowType<__bf16>
{
    static constexpr int      N = 8, kCode = kBF16;
    static constexpr uint32_t kMinusInf = 0xFF80FF80u;
    typedef row_v4u32_a2 vec_t;
    template <int E> __device__ static __forceinline__ float get(const row_v4u32& w)
    {
        return __uint_as_float(E % 2 ? w[E / 2] & 0xFFFF0000u : w[E / 2] << 16);
    }
    __device__ static __forceinline__ row_v4u32 pack(const float (&v)[8])      // to nearest even
    {
        row_v4u32 w;
#pragma unroll
        for(int i = 0; i < 4; ++i)
            w[i] = static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<__bf16>(v[2 * i])))
                   | static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<__bf16>(v[2 * i + 1]))) << 16;
        return w;
    }
};

// (STREAMED: not kept in the caches' room for what is read again.  A template's argument: of two branches that differ in it alone the
// compiler makes one ordinary access.)
template <bool STREAMED = false, typename T> __device__ __forceinline__ row_v4u32 row_load(const T* p)
{
    if constexpr(STREAMED) return __builtin_nontemporal_load(reinterpret_cast<const typename RowType<T>::vec_t*>(p));
    else                   return *reinterpret_cast<const typename RowType<T>::vec_t*>(p);
}
template <bool STREAMED = false, typename T> __device__ __forceinline__ void row_store(T* p, const row_v4u32& w)
{
    if constexpr(STREAMED) __builtin_nontemporal_store(w, reinterpret_cast<typename RowType<T>::vec_t*>(p));
    else                   *reinterpret_cast<typename RowType<T>::vec_t*>(p) = w;
}
template <typename T> __device__ __forceinline__ float row_element(const T* p) { return static_cast<float>(*p); }

// A vector of T as values, to a buffer of any type (the same for every lane); and one element.
template <typename T, bool STREAMED> __device__ __forceinline__ void vector_store(void* base, int dtype, int64_t at, const float (&v)[RowType<T>::N])
{
    if constexpr(RowType<T>::N == 8)
    {
        if(dtype == kF16) row_store<STREAMED>(static_cast<_Float16*>(base) + at, RowType<_Float16>::pack(v));
        else if(dtype == kBF16) row_store<STREAMED>(static_cast<__bf16*>(base) + at, RowType<__bf16>::pack(v));
        else
        {
            const float lo[4] = {v[0], v[1], v[2], v[3]}, hi[4] = {v[4], v[5], v[6], v[7]};
            row_store<STREAMED>(static_cast<float*>(base) + at, RowType<float>::pack(lo));
            row_store<STREAMED>(static_cast<float*>(base) + at + 4, RowType<float>::pack(hi));
        }
    }
    else if(dtype == kF32) row_store<STREAMED>(static_cast<float*>(base) + at, RowType<float>::pack(v));
    else
    {
        typedef unsigned half_vector __attribute__((ext_vector_type(2), aligned(2)));
        const float      two[8] = {v[0], v[1], v[2], v[3], 0.0f, 0.0f, 0.0f, 0.0f};
        const row_v4u32  w      = dtype == kF16 ? RowType<_Float16>::pack(two) : RowType<__bf16>::pack(two);
        *reinterpret_cast<half_vector*>(static_cast<uint16_t*>(base) + at) = half_vector{w[0], w[1]};
    }
}
__device__ __forceinline__ float element_store(void* base, int dtype, int64_t at, float v)      // returns it as stored
{
    if(dtype == kF16) return static_cast<float>(static_cast<_Float16*>(base)[at] = static_cast<_Float16>(v));
    if(dtype == kBF16) return static_cast<float>(static_cast<__bf16*>(base)[at] = static_cast<__bf16>(v));
    return static_cast<float*>(base)[at] = v;
}
template <typename T> __device__ __forceinline__ void row_decode(const row_v4u32& w, float* v)
{
    v[0] = RowType<T>::template get<0>(w); v[1] = RowType<T>::template get<1>(w);
    v[2] = RowType<T>::template get<2>(w); v[3] = RowType<T>::template get<3>(w);
    if constexpr(RowType<T>::N == 8)
    {
        v[4] = RowType<T>::template get<4>(w); v[5] = RowType<T>::template get<5>(w);
        v[6] = RowType<T>::template get<6>(w); v[7] = RowType<T>::template get<7>(w);
    }
}

// Eight consecutive elements of a row, whatever their type: what a lane of the layer norm owns.
template <typename T> struct Row8
{
    row_v4u32 w[8 / RowType<T>::N];
    __device__ __forceinline__ void load(const T* p)
    {
#pragma unroll
        for(int i = 0; i < 8 / RowType<T>::N; ++i) w[i] = row_load(p + i * RowType<T>::N);
    }
    __device__ __forceinline__ void decode(float (&v)[8]) const
    {
#pragma unroll
        for(int i = 0; i < 8 / RowType<T>::N; ++i) row_decode<T>(w[i], v + i * RowType<T>::N);
    }
    __device__ __forceinline__ void encode(const float (&v)[8])
    {
        if constexpr(RowType<T>::N == 8) w[0] = RowType<T>::pack(v);
        else
        {
            const float lo[4] = {v[0], v[1], v[2], v[3]}, hi[4] = {v[4], v[5], v[6], v[7]};
            w[0] = RowType<T>::pack(lo);
            w[1] = RowType<T>::pack(hi);
        }
    }
    __device__ __forceinline__ void store(T* p) const
    {
#pragma unroll
        for(int i = 0; i < 8 / RowType<T>::N; ++i) row_store(p + i * RowType<T>::N, w[i]);
    }
};
// ... to a buffer whose type is known at run time only (the same for every lane); `stored` receives the values as rounded
template <bool STORED> __device__ __forceinline__ void row8_store(void* base, int dtype, int64_t at, float (&v)[8])
{
    auto put = [&](auto tag) {
        typedef decltype(tag) T;
        Row8<T> r;
        r.encode(v);
        r.store(static_cast<T*>(base) + at);
        if constexpr(STORED) r.decode(v);
    };
    if(dtype == kF16) put(_Float16{});
    else if(dtype == kBF16) put(__bf16{});
    else put(float{});
}

// ---- reductions: fixed order, the result in every lane ------------------------------------------------------------------------
template <int CTRL, int ROWS = 0xF> __device__ __forceinline__ float dpp_move(float old, float v)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(old), __float_as_uint(v), CTRL, ROWS, 0xF, false));
}
constexpr int kRotate = 0x120;      // within 16 lanes, by the low digit
__device__ __forceinline__ float row16_sum(float v)
{
    v += dpp_move<kRotate + 8>(0.0f, v);
    v += dpp_move<kRotate + 4>(0.0f, v);
    v += dpp_move<kRotate + 2>(0.0f, v);
    v += dpp_move<kRotate + 1>(0.0f, v);
    return v;
}
__device__ __forceinline__ float row16_max(float v)
{
    v = fmaxf(v, dpp_move<kRotate + 8>(v, v));
    v = fmaxf(v, dpp_move<kRotate + 4>(v, v));
    v = fmaxf(v, dpp_move<kRotate + 2>(v, v));
    v = fmaxf(v, dpp_move<kRotate + 1>(v, v));
    return v;
}
__device__ __forceinline__ float lane_value(float v, int lane)
{
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}
__device__ __forceinline__ float wave64_sum(float v)
{
    v = row16_sum(v);
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}
__device__ __forceinline__ float wave64_max(float v)
{
    v = row16_max(v);
    return fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)), fmaxf(lane_value(v, 32), lane_value(v, 48)));
}

}  // namespace

}  // namespace qsync
