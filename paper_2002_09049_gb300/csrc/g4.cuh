// Weights in 4-bit integers (include/mpq.h: mpq_g4_matrix): where things lie in a tile, and eight codes' values
// as eight 16-bit floats.
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

// A word's eight values s (q - z), each rounded once to T, as four pairs in order (elements 0 and 1, 2 and 3, ..).  A code
// in the low bits of the bits of 2^k, the power whose last place is 1, is 2^k + q, so q - z is one exact difference;
// s is a bf16, which bf16 takes as it is, and fp16 from 2^-17 (the last place of its subnormals is 2^-24) to its
// largest number: there a product in T is the rounded value.  Other scales' go through fp32.
template <typename T>
struct G4Pairs;
template <>
struct G4Pairs<__nv_bfloat16> {
    static constexpr bool kBf16 = true;
    static constexpr uint32_t kPower = 0x43004300u;      // 128
    // s twice; its bits are a bf16's
    __device__ static __forceinline__ uint32_t scale(uint32_t bits) { return __byte_perm(bits, 0, 0x1010); }
    __device__ static __forceinline__ bool plain(uint32_t) { return true; }
    __device__ static __forceinline__ uint32_t whole(uint32_t v, uint32_t from) { return bits(__hsub2(as(v), as(from))); }
    __device__ static __forceinline__ uint32_t value(uint32_t v, uint32_t from, uint32_t s)
    {
        return bits(__hmul2(__hsub2(as(v), as(from)), as(s)));
    }
    // what value() rounds off, exact
    __device__ static __forceinline__ uint32_t rest(uint32_t v, uint32_t from, uint32_t s)
    {
        const __nv_bfloat162 q = __hsub2(as(v), as(from));
        return bits(__hfma2(q, as(s), __hneg2(__hmul2(q, as(s)))));
    }
    __device__ static __forceinline__ uint32_t bits(__nv_bfloat162 r) { return *reinterpret_cast<const uint32_t *>(&r); }
    __device__ static __forceinline__ __nv_bfloat162 as(uint32_t v) { return *reinterpret_cast<__nv_bfloat162 *>(&v); }
};
template <>
struct G4Pairs<__half> {
    static constexpr bool kBf16 = false;
    static constexpr uint32_t kPower = 0x64006400u;      // 1024
    __device__ static __forceinline__ uint32_t scale(uint32_t bits)
    {
        return G4Pairs::bits(__float2half2_rn(bf16_bits(bits)));
    }
    __device__ static __forceinline__ bool plain(uint32_t bits)      // |s| in [2^-17, 2^15], or 0
    {
        const uint32_t m = bits & 0x7fffu;
        return m - 0x3700u <= 0x4700u - 0x3700u || m == 0;
    }
    __device__ static __forceinline__ uint32_t whole(uint32_t v, uint32_t from) { return bits(__hsub2(as(v), as(from))); }
    __device__ static __forceinline__ uint32_t value(uint32_t v, uint32_t from, uint32_t s)
    {
        return bits(__hmul2(__hsub2(as(v), as(from)), as(s)));
    }
    __device__ static __forceinline__ uint32_t rest(uint32_t v, uint32_t from, uint32_t s)
    {
        const __half2 q = __hsub2(as(v), as(from));
        return bits(__hfma2(q, as(s), __hneg2(__hmul2(q, as(s)))));
    }
    __device__ static __forceinline__ uint32_t bits(__half2 r) { return *reinterpret_cast<const uint32_t *>(&r); }
    __device__ static __forceinline__ __half2 as(uint32_t v) { return *reinterpret_cast<__half2 *>(&v); }
};

// A group's scale and zero point as g4_values takes them.
struct G4Scale {
    uint32_t s, from, bits;
};
template <typename T>
__device__ __forceinline__ G4Scale g4_scale(uint32_t bits, uint32_t z)
{
    return {G4Pairs<T>::scale(bits), G4Pairs<T>::kPower | z | z << 16, bits};
}

// A pair of a word's codes as the bits of the power plus each: a whole number set into the last places of a power's
// significand, the conversion of Warren, Hacker's Delight, 2nd ed., 17-2.
template <typename T>
__device__ __forceinline__ uint32_t g4_pair(uint32_t w, int j)
{
    uint32_t v;                                  // (w >> 4 j) & 0x000f000f | the power: one operation of three inputs
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(v) : "r"(w >> (4 * j)), "n"(0x000f000f), "n"(G4Pairs<T>::kPower));
    return v;
}

// A word's eight q - z, whole numbers that either type holds.
template <typename T>
__device__ __forceinline__ void g4_whole(uint32_t w, uint32_t from, uint32_t (&p)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = G4Pairs<T>::whole(g4_pair<T>(w, j), from);
}

// What the word's eight values lose to their rounding: s and q - z have 8 and 4 bits, their product 12, of which bf16 keeps
// 8 and fp16 11, so what is left is a T again (where it is not below T's least place: bf16's 2^-133, fp16's 2^-24).
template <typename T>
__device__ __forceinline__ void g4_rest(uint32_t w, const G4Scale &g, uint32_t (&p)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = G4Pairs<T>::rest(g4_pair<T>(w, j), g.from, g.s);
}

// FAR: scales that G4Pairs<T>::plain does not hold for are among a warp's (hardly a matrix has such), so all of them
// go through fp32.  (A test at every word cost fp16 9.1 -> 16.2 us for 5 x 11,008 x 4,096.)
template <typename T, bool FAR>
__device__ __forceinline__ void g4_values(uint32_t w, const G4Scale &g, uint32_t (&p)[4])
{
    if constexpr (FAR) {
        const float s = bf16_bits(g.bits);
        const int z = (int)(g.from & 255u);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            p[j] = pack2((float)((int)(w >> (4 * j) & 15u) - z) * s, (float)((int)(w >> (4 * j + 16) & 15u) - z) * s, T());
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = G4Pairs<T>::value(g4_pair<T>(w, j), g.from, g.s);
    }
}

// Whether a warp has a scale, two a word, that asks for FAR.
template <typename T, int W>
__device__ __forceinline__ bool g4_far(const uint32_t (&words)[W])
{
    if (G4Pairs<T>::kBf16) return false;
    bool far = false;
#pragma unroll
    for (int i = 0; i < W; ++i) far |= !G4Pairs<T>::plain(words[i] & 0xffffu) || !G4Pairs<T>::plain(words[i] >> 16);
    return __any_sync(0xffffffffu, far) != 0;
}

}  // namespace mpq
