// Loads, stores and sums shared by the norm and dropout kernels (internal device code).
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "norm.h"

namespace sk {

template <int DT> struct Elem;
template <> struct Elem<0> { typedef float type; };
template <> struct Elem<1> { typedef __bf16 type; };
template <> struct Elem<2> { typedef _Float16 type; };
template <int DT> using elem_t = typename Elem<DT>::type;

// N elements side by side, aligned to one element only: the hardware takes global accesses of four words at any
// address, and rows or planes of odd length begin anywhere
template <int DT, int N> struct Line {
    typedef elem_t<DT> type __attribute__((ext_vector_type(N), aligned(sizeof(elem_t<DT>))));
};
template <int DT, int N> using line_t = typename Line<DT, N>::type;

// Addresses are a base that is equal in all lanes of a wave and 32 bits a lane: one register a lane instead of two, and the additions on the
// scalar unit.  `off` counts bytes.
typedef const char *src_t;
typedef char *dst_t;
// Results are stored as data that is not read again soon (nontemporal): they would push out what is still read.  Plain and so, us: norm of 65536 x 2048
// bf16 126 and 108, residual + dropout + norm of 16384 x 4096 bf16 106 and 96, norm of 48 x 527^2 fp32 27 and 23, dropout of 200 x 512^2 fp32 75 and
// 72; where everything stays in the L2 no difference (dropout of 1024 x 28^2 bf16 4.6 and 4.4).
template <int DT, int N> __device__ __forceinline__ line_t<DT, N> packed(const float (&f)[N])
{
    line_t<DT, N> v;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = static_cast<elem_t<DT>>(f[j]);
    return v;
}
template <int DT, int N> __device__ __forceinline__ void store_at(dst_t base, uint32_t off, const float (&f)[N])
{
    __builtin_nontemporal_store(packed<DT, N>(f), reinterpret_cast<line_t<DT, N> *>(base + off));
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// a * b, rounded: never part of a fused operation.  gamma * dy minus its mean has to vanish where they are equal (one channel), as it does not if one of
// the two is the unrounded product.
__device__ __forceinline__ float product(float a, float b)
{
#pragma clang fp contract(off)
    return a * b;
}

// N elements as the words that hold them, which is how they stay in registers: 16-bit ones are widened at each use
template <int DT, int N> struct Words {
    static constexpr int count = (N * (DT == 0 ? 4 : 2) + 3) / 4;
    uint32_t w[count];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < count; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void load(src_t base, uint32_t off)
    {
        if constexpr (N == 1) {
            if constexpr (DT == 0) w[0] = __float_as_uint(*reinterpret_cast<const float *>(base + off));
            else w[0] = *reinterpret_cast<const uint16_t *>(base + off);
        } else {
            typedef uint32_t Line __attribute__((ext_vector_type(count), aligned(sizeof(elem_t<DT>))));
            const Line v = *reinterpret_cast<const Line *>(base + off);
#pragma unroll
            for (int i = 0; i < count; ++i) w[i] = v[i];
        }
    }
    __device__ __forceinline__ float operator[](int i) const
    {
        if constexpr (DT == 0) return __uint_as_float(w[i]);
        else if constexpr (DT == 1) return __uint_as_float((i & 1) ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else return (float)__builtin_bit_cast(_Float16, (uint16_t)((i & 1) ? w[i / 2] >> 16 : w[i / 2]));
    }
    // the next use is to widen again, not to find the fp32 value still in a register
    __device__ __forceinline__ void forget()
    {
        if constexpr (DT != 0)
#pragma unroll
            for (int i = 0; i < count; ++i) asm volatile("" : "+v"(w[i]));
    }
};

// v + the v of the lane whose number differs in bit STEP, over lanes whose lower bits are summed already (STEP 4 and 8: mirrored
// halves, of which every lane of a half holds the same); exchanges within sixteen lanes are operand modifiers, not LDS traffic
template <int STEP> __device__ __forceinline__ float add_across(float v)
{
    if (STEP == 1) return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0xB1, 0xF, 0xF, true));      // lanes 1 0 3 2 of four
    if (STEP == 2) return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x4E, 0xF, 0xF, true));      // lanes 2 3 0 1 of four
    if (STEP == 4) return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x141, 0xF, 0xF, true));     // eight lanes mirrored
    if (STEP == 8) return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x140, 0xF, 0xF, true));     // sixteen lanes mirrored
    return v + __shfl_xor(v, STEP);
}

// sum over groups of G neighbouring lanes (G a power of two up to 64), in every lane of the group
template <int G> __device__ __forceinline__ float sum_lanes(float v)
{
    if (G > 1) v = add_across<1>(v);
    if (G > 2) v = add_across<2>(v);
    if (G > 4) v = add_across<4>(v);
    if (G > 8) v = add_across<8>(v);
    if (G > 16) v = add_across<16>(v);
    if (G > 32) v = add_across<32>(v);
    return v;
}

// sum over the lanes with equal number modulo P (P a power of two from 4 to 64), in every one of them
template <int P> __device__ __forceinline__ float sum_over_groups(float v)
{
    if (P < 8) v += __shfl_xor(v, 4);
    if (P < 16) v += __shfl_xor(v, 8);
    if (P < 32) v += __shfl_xor(v, 16);
    if (P < 64) v += __shfl_xor(v, 32);
    return v;
}

// A stretch of a line, V elements a lane in whole vectors.  Lanes whose V would reach over the stretch's end take its last V instead; what two lanes hold is
// computed alike and stored twice, by lanes of one wave, after both have read it (so results may go to the operands' place).  A stretch of the line's
// last 1 to V - 1 elements takes V, and the one in front of it ends so much earlier: no element is in two stretches.
template <int V> struct Stretch {
    long start;                                         // its first element: equal in all lanes
    uint32_t length, at;                                // the lane's first, behind that
    __device__ __forceinline__ Stretch() {}
    // the stretch of `span` from element `first` on, of a line of `count` >= V; at: lane number * V
    __device__ __forceinline__ Stretch(long first, int span, long count, uint32_t mine)
    {
        const long end = first + span;
        start = first < count - V ? first : count - V;
        length = (uint32_t)((end >= count ? count : end < count - V ? end : count - V) - start);
        at = mine < length - V ? mine : length - V;
    }
    __device__ __forceinline__ bool empty(uint32_t mine) const { return mine >= length; }
};

// This workgroup's number among gridDim.x such that neighbours run on one XCD: workgroups go to the eight XCDs in turn, each has an L2 of its own, and lines
// of maps begin anywhere, so neighbouring tiles share the cache lines at their ends.
__device__ __forceinline__ unsigned neighbour()
{
    const unsigned xcd = blockIdx.x % 8, each = gridDim.x / 8, more = gridDim.x % 8;
    return xcd * each + (xcd < more ? xcd : more) + blockIdx.x / 8;
}

// workgroups for so much work: up to 2^21 (a grid may have 2^32 - 1 threads), which then walk it
inline unsigned norm_blocks(long work, long each)
{
    const long b = (work + each - 1) / each;
    return (unsigned)(b < (1L << 21) ? b : 1L << 21);
}

// The first error of a call's launches: reading it clears it, so what a later launch reads says nothing of those before.
struct Launches {
    hipError_t first = hipSuccess;
    bool failed(hipError_t e)
    {
        if (first == hipSuccess) first = e;
        return first != hipSuccess;
    }
    bool failed() { return failed(hipGetLastError()); }         // with the launch just made
    hipError_t status() { return failed() ? first : hipSuccess; }
};

// dgamma and dbeta from the `copies` copies of their sums, each [2][c rounded up to 4]
hipError_t launch_norm_reduce(const float *scratch, int copies, float *dgamma, float *dbeta, int c, hipStream_t stream);
__host__ __device__ inline long norm_copy_floats(long c) { return 2 * ((c + 3) / 4 * 4); }

// the kernels for each order of the channels
hipError_t launch_norm_rows(const NormArgs &a, hipStream_t stream);
hipError_t launch_norm_planes(const NormArgs &a, hipStream_t stream);          // MAPS and OCTETS
int norm_rows_bwd_copies(const NormSpan &s);
int norm_planes_bwd_copies(const NormSpan &s);
hipError_t launch_norm_rows_bwd(const NormBwdArgs &a, int copies, hipStream_t stream);
hipError_t launch_norm_planes_bwd(const NormBwdArgs &a, int copies, hipStream_t stream);

}  // namespace sk
