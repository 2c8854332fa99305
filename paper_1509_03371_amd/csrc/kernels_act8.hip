// Tensors into 8 bits and back.
#include "act8_block.h"

namespace sk {

namespace {

// HBM bounds both.  A lane takes eight values of a line, four lanes a block, and a wave U times as many, all of them asked for before the first is used.
// 200 x 512^2 fp32, 264 MB either way: packed in 49 us = 5.4 TB/s, unpacked in 61 = 4.3.  fp32 results are written 32 bytes a lane, in two halves.  Unpacking alone, over
// and over, takes 84 us so, 68 with results stored plainly and 58 with four values a lane, which leave no gaps; but behind the packing, which leaves what it reads in the caches, 61, 77 and
// 75: there and back 16384 x 4096 141 us, plainly 160, and 48 x 527^2 35 and 40.  One thread a block: 2900 us both.
// LONG: a wave's values are of one line, whose place it works out on the scalar unit; a line takes as many waves as it needs.  Short lines: each lane works out
// its own.
template <bool LONG, int U> struct Octets {
    struct At {
        long b, k;               // image or row, map
        long o;                  // octet of the line
    };
    const Pack8Args &a;
    const Walk8 &w;
    long line, o0;               // LONG: of the wave; else its first octet of all
    __device__ __forceinline__ Octets(const Pack8Args &a_, const Walk8 &w_, long wave) : a(a_), w(w_)
    {
        if (LONG) {
            line = wave / w.pieces;
            o0 = (wave - line * w.pieces) * (64 * U);
        } else {
            line = 0;
            o0 = wave * (64 * U);
        }
    }
    __device__ __forceinline__ At at(int u) const
    {
        const long o = o0 + 64 * u + (threadIdx.x & 63);
        if (LONG) {
            const long b = w.maps ? line / a.c : line;
            return {b, line - b * a.c, o};
        }
        const long l = w.octets.divide(o), b = w.maps ? w.channels.divide(l) : l;
        return {b, l - b * a.c, o - l * w.octets.by};
    }
    __device__ __forceinline__ bool there(const At &p) const { return LONG ? 8 * p.o < w.length : p.b < a.n; }
};

// LANES that hold a block: four, or one where lines have eight values at most
template <int DT, int CODE, bool LONG, int U, int LANES> __global__ __launch_bounds__(256) void pack8_kernel(Pack8Args a, Walk8 w)
{
    const long step = gridDim.x * 4L;
    for (long wave = neighbour() * 4L + uniform(threadIdx.x >> 6); wave < w.waves; wave += step) {
        const Octets<LONG, U> octets(a, w, wave);
        Words<DT, 8> x[U];
        int left[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const auto p = octets.at(u);
            left[u] = octets.there(p) ? (int)std::min<long>(8, w.length - 8 * p.o) : 0;
            load_octet<DT>(static_cast<src_t>(a.x.p) + sizeof(elem_t<DT>) * (p.b * a.x.sn + (w.maps ? p.k * a.x.sc : 0) + 8 * p.o), left[u], x[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const auto p = octets.at(u);
            float f[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = x[u][j];
            uint8_t *codes = a.packed.codes + p.b * a.packed.sn + (w.maps ? p.k * a.packed.sc : 0) + 8 * p.o;
            uint8_t *scale = a.packed.scales + p.b * a.packed.ssn + (w.maps ? p.k * a.packed.ssc : 0) + p.o / 4;
            put_octet<DT, CODE, LANES>(f, left[u], codes, p.o % 4 == 0 ? scale : nullptr);
        }
    }
}

template <int DT, int CODE, bool LONG, int U> __global__ __launch_bounds__(256) void unpack8_kernel(Pack8Args a, Walk8 w)
{
    const long step = gridDim.x * 4L;
    for (long wave = neighbour() * 4L + uniform(threadIdx.x >> 6); wave < w.waves; wave += step) {
        const Octets<LONG, U> octets(a, w, wave);
        uint32_t c[U][2], scale[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const auto p = octets.at(u);
            const int left = octets.there(p) ? (int)std::min<long>(8, w.length - 8 * p.o) : 0;
            load_codes(a.packed.codes + p.b * a.packed.sn + (w.maps ? p.k * a.packed.sc : 0) + 8 * p.o, left, c[u]);
            scale[u] = left > 0 ? a.packed.scales[p.b * a.packed.ssn + (w.maps ? p.k * a.packed.ssc : 0) + p.o / 4] : 127;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const auto p = octets.at(u);
            const int left = octets.there(p) ? (int)std::min<long>(8, w.length - 8 * p.o) : 0;
            float f[8];
            octet_of_codes<CODE>(c[u], scale[u], f);
            store_octet<DT>(static_cast<dst_t>(a.x.p) + sizeof(elem_t<DT>) * (p.b * a.x.sn + (w.maps ? p.k * a.x.sc : 0) + 8 * p.o), left, f);
        }
    }
}

// Short walks and long ones, us of packing and of unpacking 2^24 bf16 values: lines of 200 14 and 12, and 33 and 30; of 256 11 and 10, and 26 and 24; of 300 16 and 18, and 26 and 25; of 512
// 11 and 10, and 13 and 12; of 1024 11 and 10 both.  fp32 lines of 300 and 400 pack faster in short walks (16, and 23 and 18) and unpack faster in long ones (28 and 23, and 25 and 17).
constexpr long kLongLine = 256;

// f(LONG, U, LANES), and the walk
template <class F> void pick_walk(const NormSpan &s, Walk8 &w, F f)
{
    w.maps = s.layout == MAPS;
    w.length = w.maps ? s.plane : s.c;
    // (lines of at most eight: one lane each.  1551889 rows of four fp16 there and back: 26 us, with four lanes a line 71.)
    const long lines = w.maps ? s.n * s.c : s.n, octets = w.length <= 8 ? 1 : 4 * blocks_of(w.length);
    auto go = [&](auto is_long, auto u, auto lanes) {
        if (is_long()) {
            w.pieces = (octets + 64 * u() - 1) / (64 * u());
            w.waves = lines * w.pieces;
        } else {
            w.octets = Divisor8(octets);
            w.channels = Divisor8(s.c);
            w.waves = (lines * octets + 64 * u() - 1) / (64 * u());
        }
        f(is_long, u, lanes);
    };
    typedef std::true_type Yes;
    typedef std::false_type No;
    typedef std::integral_constant<int, 1> One;
    typedef std::integral_constant<int, 2> Two;
    typedef std::integral_constant<int, 4> Four;
    // (1310 x 200 2.7 us, with two octets a lane 3.4)
    const bool few = lines * octets < 64 * 1024;
    if (w.length <= 8) return few ? go(No{}, One{}, One{}) : go(No{}, Two{}, One{});
    if (w.length <= kLongLine) return few ? go(No{}, One{}, Four{}) : go(No{}, Two{}, Four{});
    // so that few pieces are left half empty
    if (octets <= 64) return go(Yes{}, One{}, Four{});
    // (256 x 4096 2.8 us with two octets a lane, 3.7 with four; 16384 x 4096 bf16 unpacked in 33.8 and 31.5, but 2048 x 4096 fp32 packed in 8.5 and 10.2, unpacked in 11 and 16)
    if (octets <= 128 || lines * octets < 64 * 4096) return go(Yes{}, Two{}, Four{});
    return go(Yes{}, Four{}, Four{});
}

template <class F> void pick_dtype(int dtype, F f)
{
    if (dtype == 0) return f(std::integral_constant<int, 0>{});
    if (dtype == 1) return f(std::integral_constant<int, 1>{});
    return f(std::integral_constant<int, 2>{});
}

}  // namespace

hipError_t launch_pack8(const Pack8Args &a, hipStream_t stream)
{
    Walk8 w;
    pick_walk(a, w, [&](auto is_long, auto u, auto lanes) {
        pick_dtype(a.dtype, [&](auto dt) {
            pick_code(a.packed.code, [&](auto code) { pack8_kernel<dt(), code(), is_long(), u(), lanes()><<<norm_blocks(w.waves, 4), 256, 0, stream>>>(a, w); });
        });
    });
    return hipGetLastError();
}

hipError_t launch_unpack8(const Pack8Args &a, hipStream_t stream)
{
    Walk8 w;
    pick_walk(a, w, [&](auto is_long, auto u, auto) {
        pick_dtype(a.dtype, [&](auto dt) {
            pick_code(a.packed.code, [&](auto code) { unpack8_kernel<dt(), code(), is_long(), u()><<<norm_blocks(w.waves, 4), 256, 0, stream>>>(a, w); });
        });
    });
    return hipGetLastError();
}

}  // namespace sk
