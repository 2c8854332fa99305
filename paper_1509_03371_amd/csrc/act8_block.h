// Eight values of a line, four lanes a block in 8 bits (internal device code).
#pragma once
#include "act8_device.h"

namespace sk {

// Division of numbers below 2^31 by one below 2^31, rounded down: i m >> s with m = ceil(2^s / d), s = 31 + ceil(log2 d), is exact for them (m d exceeds 2^s
// by less than d <= 2^(s-31), and so i m / 2^s exceeds i / d by less than 1 / d).  Larger numbers are divided as they are.
struct Divisor8 {
    long by = 1;
    uint32_t m = 0;
    int s = 0;
    Divisor8() {}
    explicit Divisor8(long d) : by(d)
    {
        if (d >= 1L << 31) return;
        s = 31;
        while (1L << (s - 31) < d) ++s;
        m = (uint32_t)((((unsigned __int128)1 << s) + d - 1) / d);
    }
    __device__ __forceinline__ long divide(long i) const
    {
        if ((uint64_t)i < 1u << 31 && s) return (long)(((uint64_t)m * (uint32_t)i) >> s);
        return i / by;
    }
};

struct Walk8 {
    bool maps;
    long length;                 // of a line
    long waves;                  // waves' worth of it all
    long pieces;                 // of a long line
    Divisor8 octets, channels;
};

// the first `left` of eight elements, zeros behind them (left <= 0: none, left >= 8: all)
template <int DT> __device__ __forceinline__ void load_octet(src_t p, int left, Words<DT, 8> &w)
{
    if (left >= 8) {
        w.load(p, 0);
        return;
    }
    w.clear();
#pragma unroll
    for (int j = 0; j < 7; ++j)
        if (j < left) {
            if constexpr (DT == 0) w.w[j] = *reinterpret_cast<const uint32_t *>(p + 4 * j);
            else w.w[j / 2] |= (uint32_t)*reinterpret_cast<const uint16_t *>(p + 2 * j) << 16 * (j & 1);
        }
}
template <int DT> __device__ __forceinline__ void store_octet(dst_t p, int left, const float (&f)[8])
{
    if (left >= 8) {
        store_at<DT, 8>(p, 0, f);
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < left) store_at<DT, 1>(p, sizeof(elem_t<DT>) * j, {f[j]});
    }
}

typedef uint32_t codes2 __attribute__((ext_vector_type(2), aligned(1)));
__device__ __forceinline__ void load_codes(const uint8_t *p, int left, uint32_t (&c)[2])
{
    if (left >= 8) {
        const codes2 v = *reinterpret_cast<const codes2 *>(p);
        c[0] = v[0];
        c[1] = v[1];
        return;
    }
    c[0] = c[1] = 0;
#pragma unroll
    for (int j = 0; j < 7; ++j)
        if (j < left) c[j / 4] |= (uint32_t)p[j] << 8 * (j & 3);
}
template <int CODE> __device__ __forceinline__ void octet_of_codes(const uint32_t (&c)[2], uint32_t byte, float (&f)[8])
{
    const float scale = Code8<CODE>::scale(byte);
    float lo[4], hi[4];
    Code8<CODE>::values(c[0], scale, lo);
    Code8<CODE>::values(c[1], scale, hi);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f[j] = lo[j];
        f[4 + j] = hi[j];
    }
}

// v, or the v of the lane whose number differs in bit STEP, whichever is larger
template <int STEP> __device__ __forceinline__ uint32_t max_across(uint32_t v)
{
    const uint32_t o = STEP == 1 ? __builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, true) : __builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, true);
    return v > o ? v : o;
}
template <int LANES> __device__ __forceinline__ uint32_t max_of_block(uint32_t v)
{
    static_assert(LANES == 1 || LANES == 4, "a block is one lane's or four neighbours'");
    if (LANES == 1) return v;
    return max_across<2>(max_across<1>(v));
}

// A block whose values are all finite and within the limit needs no look at each of them: that is told by its largest magnitude's bits.
template <int DT, int CODE, int LANES> __device__ __forceinline__ uint32_t codes_of_octet(const float (&f)[8], uint32_t (&c)[2])
{
    constexpr uint32_t limit = Code8<CODE>::limit(DT);
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t m = magnitude(f[j]);
        most = most > m ? most : m;
    }
    most = max_of_block<LANES>(most);
    if (most <= limit) {
        const uint32_t byte = Code8<CODE>::scale_byte(most);
        const float inverse = Code8<CODE>::inverse(byte);
        c[0] = Code8<CODE>::four(f[0], f[1], f[2], f[3], inverse);
        c[1] = Code8<CODE>::four(f[4], f[5], f[6], f[7], inverse);
        return byte;
    }
    most = 0;                    // (the lanes of a block come here together)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t m = counted(f[j], limit);
        most = most > m ? most : m;
    }
    most = max_of_block<LANES>(most);
    const uint32_t byte = Code8<CODE>::scale_byte(most);
    c[0] = c[1] = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) c[j / 4] |= any_code<CODE>(f[j], Code8<CODE>::inverse(byte), limit) << 8 * (j & 3);
    return byte;
}

// A lane's eight values in 8 bits: the first `left` to `codes`, and the block's scale to `scale` if there is one and any value of it.  Values behind `left` are
// zeros.  All lanes of a block come here.
template <int DT, int CODE, int LANES> __device__ __forceinline__ void put_octet(const float (&f)[8], int left, uint8_t *codes, uint8_t *scale)
{
    uint32_t c[2];
    const uint32_t byte = codes_of_octet<DT, CODE, LANES>(f, c);
    if (left >= 8) {
        const codes2 v = {c[0], c[1]};
        __builtin_nontemporal_store(v, reinterpret_cast<codes2 *>(codes));
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < left) codes[j] = (uint8_t)(c[j / 4] >> 8 * (j & 3));
    }
    if (scale && left > 0) *scale = (uint8_t)byte;
}

}  // namespace sk
