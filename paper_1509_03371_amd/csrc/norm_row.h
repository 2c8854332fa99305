// Rows of channels side by side: which lanes hold what of them (internal device code of the norm kernels).
#pragma once
#include "norm_device.h"

namespace sk {

// A row belongs to G lanes; lane l holds channels 8*(k*G + l) .. + 7 for k < K, the whole row in registers: one read of every input, one write of
// every output, and the variance from the values themselves about their mean (no sum of squares to cancel).  Eight channels a lane because that is
// what one call of dropout's generator serves; 16 bytes a load in 16 bits, two loads in fp32.  Rows of up to 64 lanes' worth need no LDS; longer ones
// add their waves' sums there.
template <int DT, int G> struct Row {
    typedef elem_t<DT> E;
    static constexpr int S = sizeof(E);
    static constexpr bool SHORT = G == 1 || G == 64;    // may have rows of fewer than eight (64: rows too far apart for other G)
    const int c;
    const int lane, sub;                                // of the row's G; row among the wave's

    __device__ __forceinline__ explicit Row(int c_) : c(c_), lane(threadIdx.x % G), sub(G < 64 ? (threadIdx.x & 63) / G : 0) {}
    __device__ __forceinline__ int channel(int k) const { return 8 * (k * G + lane); }
    // eight elements of a line of c, aligned to one of them.  A lane whose eight would reach over the line's end reads its last eight instead (lanes behind
    // the end too): `fit` then puts them in place.
    template <int D> __device__ __forceinline__ void load(src_t p, uint32_t off, int k, Words<D, 8> &w) const
    {
        constexpr int size = sizeof(elem_t<D>);
        if (SHORT && c < 8) {                           // lines of fewer than eight elements, one by one
            w.clear();
            if (channel(k) == 0)
#pragma unroll
                for (int j = 0; j < 7; ++j)
                    if (j < c) {
                        if constexpr (D == 0) w.w[j] = *reinterpret_cast<const uint32_t *>(p + off + 4 * j);
                        else w.w[j / 2] |= (uint32_t)*reinterpret_cast<const uint16_t *>(p + off + 2 * j) << 16 * (j & 1);
                    }
        } else {
            w.load(p, off + size * std::min(channel(k), c - 8));
        }
    }
    // zeros behind the line's end; `exact`: there is nothing behind it
    template <int D> __device__ __forceinline__ void fit(int k, bool exact, Words<D, 8> &w) const
    {
        constexpr int n = Words<D, 8>::count;
        if (exact || (SHORT && c < 8)) return;
        const int left = c - channel(k);
        if (c % 8) {                                    // down by 8 - c % 8 elements in the one lane that read over the end
            const bool tail = left > 0 && left < 8;
            const int down = 8 - c % 8;
            auto words = [&](int by) {
#pragma unroll
                for (int i = 0; i < n; ++i) w.w[i] = tail ? (i + by < n ? w.w[i + by < n ? i + by : 0] : 0) : w.w[i];
            };
            if (down & 4) words(n / 2);
            if (down & 2) words(n / 4);
            if (down & 1) {
                if constexpr (D == 0) {
                    words(1);
                } else {
#pragma unroll
                    for (int i = 0; i < n; ++i) w.w[i] = tail ? (i + 1 < n ? __builtin_amdgcn_alignbit(w.w[i + 1 < n ? i + 1 : 0], w.w[i], 16) : w.w[i] >> 16) : w.w[i];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < n; ++i) w.w[i] = left > 0 ? w.w[i] : 0;
    }
    // row: the first of the wave's
    __device__ __forceinline__ src_t from(const NormView &v, long row) const { return static_cast<src_t>(v.p) + S * row * v.sn; }
    __device__ __forceinline__ uint32_t offset(const NormView &v) const { return G < 64 ? (uint32_t)sub * (uint32_t)(S * v.sn) : 0; }
    // PLAIN: as data that may be read again soon
    template <bool PLAIN = false> __device__ __forceinline__ void store(const NormView &v, long row, int k, const float (&f)[8]) const
    {
        const int left = c - channel(k);
        const dst_t p = static_cast<dst_t>(v.p) + S * row * v.sn;
        const uint32_t off = offset(v) + S * channel(k);
        if (PLAIN && left >= 8) {
            *reinterpret_cast<line_t<DT, 8> *>(p + off) = packed<DT, 8>(f);
        } else if (left >= 8) {
            store_at<DT, 8>(p, off, f);
        } else if (left > 0) {                          // c % 8 elements, by four, two and one
            const int r = c % 8;
            auto one = [&](float a, float b, float c_, float d) { return (r & 4) ? ((r & 2) ? d : c_) : (r & 2) ? b : a; };       // (values, no places)
            auto two = [&](float a, float b) { return (r & 4) ? b : a; };
            if (r & 4) store_at<DT, 4>(p, off, {f[0], f[1], f[2], f[3]});
            if (r & 2) store_at<DT, 2>(p, off + S * (r & 4), {two(f[0], f[4]), two(f[1], f[5])});
            if (r & 1) store_at<DT, 1>(p, off + S * (r & 6), {one(f[0], f[2], f[4], f[6])});
        }
    }
};

// sum over a row's lanes, in every one of them
template <int G> struct RowSum {
    float *part;                 // G > 64: two halves of G / 64 floats
    int half = 0;
    __device__ __forceinline__ float operator()(float v)
    {
        v = sum_lanes<(G < 64 ? G : 64)>(v);
        if (G <= 64) return v;
        constexpr int W = G / 64;
        float *p = part + half * W;
        half ^= 1;               // the next sum goes to the other half: one barrier a sum
        if ((threadIdx.x & 63) == 0) p[threadIdx.x >> 6] = v;
        __syncthreads();
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) s += p[i];
        return s;
    }
};

// the first row of this wave; G > 64: of the workgroup
template <int G, int T> __device__ __forceinline__ long first_row()
{
    if (G > 64) return blockIdx.x;
    return (blockIdx.x * (long)(T / 64) + uniform(threadIdx.x >> 6)) * (64 / G);
}
template <int G, int T> __device__ __forceinline__ long row_step() { return G > 64 ? gridDim.x : gridDim.x * (long)(T / G); }

inline bool far_apart(std::initializer_list<const NormView *> views)
{
    for (const NormView *v : views)
        if (v->p && v->sn >= (1L << 24)) return true;   // 64 rows of elements of at most four bytes
    return false;
}

}  // namespace sk
