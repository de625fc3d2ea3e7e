// Rows of matrices in fp32 or bf16, as the training operators' kernels read, add up and write them.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

namespace gp {

typedef unsigned short bf16_t;

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16_t v) { return __uint_as_float((unsigned)v << 16); }
template <typename T>
__device__ __forceinline__ T narrow(float v)
{
    if constexpr (std::is_same<T, float>::value)
        return v;
    else
        return __builtin_bit_cast(bf16_t, (__bf16)v);  // to nearest even
}

// N elements from or to any element's boundary: gfx950 loads and stores vectors from there in one request
template <typename T, int N>
struct Vec {
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <typename T>
struct Vec<T, 1> {
    typedef T type;
};
// element i of one, widened
template <typename T, int N>
__device__ __forceinline__ float element(const typename Vec<T, N>::type& x, int i)
{
    if constexpr (N == 1)
        return widen(x);
    else
        return widen(x[i]);
}
template <typename T, int N>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[N])
{
    if constexpr (N == 1) {
        v[0] = widen(*p);
    } else {
        const typename Vec<T, N>::type x = *reinterpret_cast<const typename Vec<T, N>::type*>(p);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = widen(x[i]);
    }
}
template <typename T, int N>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[N])
{
    if constexpr (N == 1) {
        *p = narrow<T>(v[0]);
    } else {
        typename Vec<T, N>::type x;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = narrow<T>(v[i]);
        *reinterpret_cast<typename Vec<T, N>::type*>(p) = x;
    }
}

// row number i of a list of 32 or 64 bits each
__device__ __forceinline__ int64_t token_at(const void* tokens, int wide, int64_t i)
{
    return wide ? ((const int64_t*)tokens)[i] : (int64_t)((const int32_t*)tokens)[i];
}

// All lanes of a team of W (a power of two up to 64, on a multiple of W) get the team's result, the same bits each.  Up to 16 lanes a step is a move inside the
// instruction that uses it: neighbours, pairs, then mirrored halves (which hold the same by then); beyond, rows of 16 and halves of 32 change places.
template <int CTRL>
__device__ __forceinline__ unsigned moved(unsigned v)
{
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
template <int CTRL>
__device__ __forceinline__ float moved(float v)
{
    return __uint_as_float(moved<CTRL>(__float_as_uint(v)));
}
template <int W, typename Op>
__device__ __forceinline__ float team(float v, Op op)
{
    static_assert(W >= 1 && W <= 64 && (W & (W - 1)) == 0, "a team is 1 to 64 lanes");
    if constexpr (W >= 2) v = op(v, moved<0xB1>(v));
    if constexpr (W >= 4) v = op(v, moved<0x4E>(v));
    if constexpr (W >= 8) v = op(v, moved<0x141>(v));
    if constexpr (W >= 16) v = op(v, moved<0x140>(v));
    if constexpr (W >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    if constexpr (W >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return v;
}
template <int W>
__device__ __forceinline__ float team_sum(float v)
{
    return team<W>(v, [](float a, float b) {
#pragma clang fp contract(off)  // (a product that one lane adds in one instruction and its neighbour in two gives them different bits)
        return a + b;
    });
}
template <int W>
__device__ __forceinline__ float team_max(float v)
{
    return team<W>(v, [](float a, float b) { return fmaxf(a, b); });
}

}  // namespace gp
