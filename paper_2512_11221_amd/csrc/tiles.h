// What the kernels over tiles of 32 query rows share (prompt.hip, draft.hip): vector types,
// bounded loads, and the treatment of values that are not finite.
#pragma once

#include <hip/hip_runtime.h>
#include <type_traits>

namespace asrkf {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4* lds_shortx4;

constexpr int kBufferFlags = 0x00020000;      // raw buffer, 32-bit data

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* p, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, bytes, kBufferFlags);
}
__device__ __forceinline__ intx4 load16(__amdgpu_buffer_rsrc_t r, int off) {
    return __builtin_bit_cast(intx4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
}

template <int N, typename F>
__device__ __forceinline__ void unroll(F f) {
    if constexpr (N > 0) {
        unroll<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

// x with 0 in the place of infinities and NaNs; bad says whether there were any
template <bool BF16>
__device__ __forceinline__ intx4 finite_part(intx4 x, bool& bad) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (BF16) {
            const bool lo = (x[i] & 0x7F80) == 0x7F80, hi = (x[i] & 0x7F800000) == 0x7F800000;
            bad |= lo || hi;
            x[i] &= (lo ? 0 : 0xFFFF) | (hi ? 0 : (int)0xFFFF0000);
        } else {
            const bool is = (x[i] & 0x7F800000) == 0x7F800000;
            bad |= is;
            x[i] = is ? 0 : x[i];
        }
    }
    return x;
}

}  // namespace asrkf
