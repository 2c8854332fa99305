// The numbers behind dropout (internal device code).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sk {

// a ^ b ^ c in one instruction (the compiler takes two)
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }

// Philox4x32-10 (J. Salmon, M. Moraes, R. Dror, D. Shaw: Parallel random numbers: as easy as 1, 2, 3; SC 2011): ten rounds
// of two 32 x 32 -> 64 bit products on a 128-bit counter, under a 64-bit key.  Every counter value gives four words that do
// not depend on any other call, so a mask can be made again wherever it is needed and is never stored.
__device__ __forceinline__ void philox4x32(uint32_t (&w)[4], uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * w[0], b = (uint64_t)0xCD9E8D57u * w[2];
        w[0] = xor3((uint32_t)(b >> 32), w[1], k0);
        w[1] = (uint32_t)b;
        w[2] = xor3((uint32_t)(a >> 32), w[3], k1);
        w[3] = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

// Which elements dropout keeps.  Sixteen bits an element: one call serves eight channels of a position, which keeps the
// products below the time of the memory traffic; the rate is a multiple of 2^-16 and the scale the exact inverse of the rate kept, so the
// expectation is exact for the rate as rounded.
struct DropMask {
    uint32_t thresh = 0;         // of 65536 numbers those below it drop an element; 0 = dropout is off
    float scale = 1.f;           // 65536 / (65536 - thresh); 0 where nothing is kept
    uint64_t seed = 0, offset = 0;
    const uint64_t *step = nullptr;   // optional, DEVICE: added to offset
    __device__ __forceinline__ uint64_t base() const { return step ? offset + *step : offset; }
};

// the numbers of channels 8*group .. 8*group + 7 of a position, low half of each word first
__device__ __forceinline__ void mask_words(uint32_t (&w)[4], const DropMask &m, uint64_t base, uint64_t position, uint32_t group)
{
    w[0] = (uint32_t)position;
    w[1] = group | (uint32_t)(position >> 32) << 24;
    w[2] = (uint32_t)base;
    w[3] = (uint32_t)(base >> 32);
    philox4x32(w, (uint32_t)m.seed, (uint32_t)(m.seed >> 32));
}

// a dropped element is a zero whatever it was (infinite and NaN ones too)
__device__ __forceinline__ float dropped(float v, const uint32_t (&w)[4], int j, const DropMask &m)
{
    const uint32_t u = (j & 1) ? w[j >> 1] >> 16 : w[j >> 1] & 0xffffu;
    return u >= m.thresh ? v * m.scale : 0.f;
}

}  // namespace sk
