// Loads and stores past the caches.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pifa {

// Loads and stores of values that nothing reads again soon: they leave the caches to
// the others, and long streams of reads and writes run faster.  Units of 4, 8 or 16
// bytes at any address.
template <int BYTES>
struct Streamed;
template <>
struct Streamed<4> {
    typedef uint32_t V __attribute__((aligned(1)));
};
template <>
struct Streamed<8> {
    typedef uint32_t V __attribute__((ext_vector_type(2), aligned(1)));
};
template <>
struct Streamed<16> {
    typedef uint32_t V __attribute__((ext_vector_type(4), aligned(1)));
};
template <typename R>
__device__ __forceinline__ R load_streamed(const void* p) {
    typedef typename Streamed<sizeof(R)>::V V;
    return __builtin_bit_cast(R, __builtin_nontemporal_load(reinterpret_cast<const V*>(p)));
}
template <typename R>
__device__ __forceinline__ void store_streamed(void* p, const R& v) {
    typedef typename Streamed<sizeof(R)>::V V;
    const V u = __builtin_bit_cast(V, v);
    __builtin_nontemporal_store(u, reinterpret_cast<V*>(p));
}

}  // namespace pifa
