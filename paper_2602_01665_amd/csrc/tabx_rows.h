// Rows of the learner's arrays: elements of three types at any alignment of theirs, in 32 bits in
// registers, and sums over the lanes that share a row.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tabx.h"

namespace tabx {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

template <int TYPE> struct Element;
template <> struct Element<TABX_F32> { typedef float one; typedef f32x4 four; };
template <> struct Element<TABX_BF16> { typedef __bf16 one; typedef bf16x4 four; };
template <> struct Element<TABX_F16> { typedef _Float16 one; typedef f16x4 four; };

// Four elements from `at` on, wherever that lies: the memory pipeline takes vectors at any address, so rows of odd
// widths and strides need no form of their own.
template <int TYPE>
__device__ __forceinline__ f32x4 load_four(const typename Element<TYPE>::one *at)
{
    typename Element<TYPE>::four v;
    __builtin_memcpy(&v, at, sizeof v);
    return __builtin_convertvector(v, f32x4);
}

// To the element's type: one rounding, to nearest even.  STREAM: past the caches.
template <int TYPE, bool STREAM = false>
__device__ __forceinline__ void store_four(typename Element<TYPE>::one *at, f32x4 v)
{
    typedef typename Element<TYPE>::four Four;
    typedef Four Anywhere __attribute__((aligned(2)));
    const Four r = __builtin_convertvector(v, Four);
    if (STREAM) __builtin_nontemporal_store(r, (Anywhere *)at);
    else __builtin_memcpy(at, &r, sizeof r);
}

// Sum over each aligned run of LANES lanes (a power of two up to 64), in all of its lanes: inside sixteen lanes
// by data-parallel moves, which need no LDS, then by swapping rows of sixteen and halves of the wavefront.
template <int PATTERN>
__device__ __forceinline__ float moved(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), PATTERN, 0xf, 0xf, true));
}

template <int LANES>
__device__ __forceinline__ float lanes_sum(float v)
{
    if (LANES >= 2) v += moved<0xB1>(v);        // quad_perm 1 0 3 2
    if (LANES >= 4) v += moved<0x4E>(v);        // quad_perm 2 3 0 1
    if (LANES >= 8) v += moved<0x141>(v);       // row_half_mirror: the other quad of eight
    if (LANES >= 16) v += moved<0x140>(v);      // row_mirror: the other eight of sixteen
    if (LANES >= 32) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    if (LANES >= 64) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return v;
}

} // namespace tabx
