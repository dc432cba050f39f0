// What the paged cache's kernels share.
#pragma once

#include <type_traits>

#include "cache.h"
#include "common.h"
#include "proxyattn.h"

namespace pa {

// Number of sequences that end at or before token t, which is t's sequence
// (s.b or more: behind the last one).  A whole wave looks at 64 ends at a
// time, up to 4096 sequences in two looks; any contents give 0 .. b.
__device__ __forceinline__ int seq_of_token(const int* starts, int b, int t) {
    const int lane = threadIdx.x & 63;
    int base = 0, step = b;
    if (b > 64) {
        step = (b + 63) / 64;
        const int last = (lane + 1) * step;
        base = step * __popcll(__ballot(last <= b && starts[min(last, b)] <= t));
        step = min(step, b - base);
    }
    return base + __popcll(__ballot(lane < step && starts[min(base + lane + 1, b)] <= t));
}

// Two values rounded to bf16 (nearest, ties to even), the first low, by the
// hardware's conversion.
__device__ __forceinline__ uint32_t pack_rne(float lo, float hi) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const f32x2 x = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// The eight 4-bit values of a word.
__device__ __forceinline__ void fp4_values(uint32_t w, float scale, float (&z)[8]) {
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0);
    const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
    const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2);
    const auto d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    z[0] = a[0], z[1] = a[1], z[2] = b[0], z[3] = b[1];
    z[4] = c[0], z[5] = c[1], z[6] = d[0], z[7] = d[1];
}

// Orders this wave's LDS accesses before and after it (a region that no other
// wave touches).
__device__ __forceinline__ void wave_lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <typename T> struct TypeTag { typedef T type; };

// Calls f with the element type, head dim and cache type as types.
template <typename F> void by_cache_type(const CacheShape& s, F f) {
    auto with_d = [&](auto t) {
        auto with_fp4 = [&](auto d) {
            if (s.fp4)
                f(t, d, std::true_type());
            else
                f(t, d, std::false_type());
        };
        if (s.d == 64)
            with_fp4(std::integral_constant<int, 64>());
        else
            with_fp4(std::integral_constant<int, 128>());
    };
    if (s.dtype == PROXYATTN_BF16)
        with_d(TypeTag<bf16>());
    else
        with_d(TypeTag<float>());
}

}  // namespace pa
