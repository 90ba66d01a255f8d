// Elements of 32 and 16 bits as the operators of the training step read and write them: vectors of 16 bytes, arithmetic in fp32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rapidgnn.h"

namespace rg {

typedef _Float16 f16;
typedef __bf16 bf16;

inline uint32_t element_bytes(uint32_t type) { return type == RG_F32 ? 4u : type == RG_BF16 || type == RG_F16 ? 2u : 0u; }

// V consecutive elements at any address that suits one element: global memory takes vector accesses at every phase (the compiler
// targets the unaligned access mode that the HSA runtime sets), so that odd widths and padded rows alike go in 16-byte accesses.
template <typename T, int V> struct PackOf { typedef T type __attribute__((ext_vector_type(V))); };
template <typename T> struct PackOf<T, 1> { typedef T type; };

template <typename T, int V> __device__ __forceinline__ typename PackOf<T, V>::type load_raw(const T *p)
{
    typedef typename PackOf<T, V>::type P __attribute__((aligned(alignof(T))));
    return *reinterpret_cast<const P *>(p);
}
template <typename T, int V> __device__ __forceinline__ void unpack(const typename PackOf<T, V>::type &raw, float (&v)[V])
{
    if constexpr (V == 1) {
        v[0] = (float)raw;
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = (float)raw[e];
    }
}
template <typename T, int V> __device__ __forceinline__ void load_pack(const T *p, float (&v)[V]) { unpack<T, V>(load_raw<T, V>(p), v); }

template <typename T, int V>
__device__ __forceinline__ void store_pack(T *p, const float (&v)[V])
{
    typedef typename PackOf<T, V>::type P __attribute__((aligned(alignof(T))));
    if constexpr (V == 1) {
        *p = (T)v[0];
    } else {
        P raw;
#pragma unroll
        for (int e = 0; e < V; ++e) raw[e] = (T)v[e];
        *reinterpret_cast<P *>(p) = raw;
    }
}

// The sum over groups of LANES lanes (a power of two up to 64), in every lane of the group.  Within 16 lanes by moves inside the
// vector unit: neighbours, pairs, then the row's halves and the row mirrored.
template <int CTRL> __device__ __forceinline__ float dpp_move(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
template <int LANES> __device__ __forceinline__ float lanes_sum(float v)
{
    static_assert(LANES == 8 || LANES == 16 || LANES == 32 || LANES == 64, "");
    v += dpp_move<0xB1>(v);                        // quad_perm 1 0 3 2
    v += dpp_move<0x4E>(v);                        // quad_perm 2 3 0 1
    v += dpp_move<0x141>(v);                       // row_half_mirror
    if constexpr (LANES >= 16) v += dpp_move<0x140>(v);      // row_mirror
    if constexpr (LANES >= 32) v += __shfl_xor(v, 16);
    if constexpr (LANES >= 64) v += __shfl_xor(v, 32);
    return v;
}

}  // namespace rg
