// Weights in 4-bit integers (include/mpq.h: mpq_g4_matrix): where things lie in a tile, and eight codes as
// eight 16-bit floats.
#pragma once

#include "elements.cuh"
#include "mpq_internal.cuh"

namespace mpq {

constexpr int G4_CODES = 1024;               // bytes of a tile's codes: 16 rows of 64
constexpr int G4_ZERO = 8;                   // the zero point of matrices without

// Byte of the word of elements 8 n .. 8 n + 7 (n = 0..15) within a row of a tile.
__host__ __device__ __forceinline__ int g4_word(int n) { return 16 * (n & 3) + 4 * (n >> 2); }

// Bit of element e (0..7) within its word.
__host__ __device__ __forceinline__ int g4_shift(int e) { return 4 * (e >> 1) + 16 * (e & 1); }

__device__ __forceinline__ float bf16_bits(uint32_t low) { return __uint_as_float(low << 16); }

// q - z of a word's eight codes, exact, as four pairs of T in order (elements 0 and 1, 2 and 3, ..): a code in the low
// bits of the bits of 2^k, the power whose last place is 1, is 2^k + q, and `from` holds 2^k + z twice.
template <typename T>
struct G4Pairs;
template <>
struct G4Pairs<__nv_bfloat16> {
    static constexpr uint32_t kPower = 0x43004300u;      // 128
    __device__ static __forceinline__ uint32_t less(uint32_t w, uint32_t from)
    {
        const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&w),
                                         *reinterpret_cast<const __nv_bfloat162 *>(&from));
        return *reinterpret_cast<const uint32_t *>(&r);
    }
};
template <>
struct G4Pairs<__half> {
    static constexpr uint32_t kPower = 0x64006400u;      // 1024
    __device__ static __forceinline__ uint32_t less(uint32_t w, uint32_t from)
    {
        const __half2 r = __hsub2(*reinterpret_cast<const __half2 *>(&w),
                                  *reinterpret_cast<const __half2 *>(&from));
        return *reinterpret_cast<const uint32_t *>(&r);
    }
};

template <typename T>
__device__ __forceinline__ uint32_t g4_from(uint32_t z) { return G4Pairs<T>::kPower | z | z << 16; }

template <typename T>
__device__ __forceinline__ void g4_pairs(uint32_t w, uint32_t from, uint32_t (&p)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t v;                          // (w >> 4 j) & 0x000f000f | the power: one operation of three inputs
        asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(v) : "r"(w >> (4 * j)), "n"(0x000f000f), "n"(G4Pairs<T>::kPower));
        p[j] = G4Pairs<T>::less(v, from);
    }
}

}  // namespace mpq
