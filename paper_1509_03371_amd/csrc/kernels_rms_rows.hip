// Root-mean-square norm of rows: the channels of a position side by side.
#include "norm_row.h"
#include "rms.h"

namespace sk {

namespace {

// Four neighbouring lanes of a row hold a block of 32 channels; rows of up to eight are one lane's.
template <int G> constexpr int block_lanes = G == 1 ? 1 : 4;

// All lanes of a block come here, those behind the row's end with zeros.  row0: the first of the wave's.
template <int DT, int G> __device__ __forceinline__ void pack_row(const Row<DT, G> &r, const PackedView &v, long row0, int k, const float (&f)[8])
{
    const int c0 = r.channel(k);
    uint8_t *codes = v.codes + row0 * v.sn + ((G < 64 ? (uint32_t)r.sub * (uint32_t)v.sn : 0) + (uint32_t)c0);
    uint8_t *scale = v.scales + row0 * v.ssn + ((G < 64 ? (uint32_t)r.sub * (uint32_t)v.ssn : 0) + (uint32_t)c0 / 32);
    put_packed<DT, block_lanes<G>>(v, f, r.c - c0, codes, c0 % 32 == 0 ? scale : nullptr);
}

// fp32 lanes write 32 bytes in two halves, which leave gaps that only a cache closes: gradient of 16384 x 4096 193 us nontemporal and 154 plain, norm of 65536 x 1000 112 and
// 102; 16 bits leave none.
template <int DT, int G> __device__ __forceinline__ void put_line(const Row<DT, G> &r, const NormView &v, long row0, int k, const float (&f)[8])
{
    r.template store<DT == 0>(v, row0, k, f);
}

// y of an octet from its s
template <int DT, int G> __device__ __forceinline__ void put_row(const Row<DT, G> &r, const RmsArgs &a, long row0, int k, bool exact, float rstd, const float (&s)[8])
{
    if (a.sum.p) put_line(r, a.sum, row0, k, s);
    if (a.sum8.codes) pack_row(r, a.sum8, row0, k, s);
    if (!a.y.p && !a.y8.codes) return;
    float o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = s[j] * rstd;
    if (a.gamma) {
        Words<0, 8> g;
        r.load(reinterpret_cast<src_t>(a.gamma), 0, k, g);
        r.fit(k, exact, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] *= g[j];
    }
    if (a.y.p) put_line(r, a.y, row0, k, o);
    if (a.y8.codes) pack_row(r, a.y8, row0, k, o);
}

// G lanes hold a row, K octets each: one read and one write.  Squares need no mean taken off, so the sum of them is the one sum there is.  HBM bounds it: residual,
// sum and e4m3 result of 16384 x 4096 bf16, 471 MB in 84 us = 5.6 TB/s; 16 x 1024 bf16 3.8 us, a launch.
template <int DT, int G, int K, int T> __global__ __launch_bounds__(T) void rms_rows_kernel(RmsArgs a)
{
    __shared__ float part[G > 64 ? 2 * (G / 64) : 1];
    RowSum<G> total{part};
    const Row<DT, G> r(a.c);
    const bool exact = a.c == 8 * G * K;
    for (long row0 = first_row<G, T>(); row0 < a.n; row0 += row_step<G, T>()) {     // (G > 64: every thread alike)
        const long row = row0 + r.sub;
        if (G < 64 && row >= a.n) break;
        float s[K][8];
        Words<DT, 8> x[K], u[K];
#pragma unroll
        for (int k = 0; k < K; ++k) r.load(r.from(a.x, row0), r.offset(a.x), k, x[k]);
        if (a.residual.p)
#pragma unroll
            for (int k = 0; k < K; ++k) r.load(r.from(a.residual, row0), r.offset(a.residual), k, u[k]);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            r.fit(k, exact, x[k]);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[k][j] = x[k][j];
        }
        if (a.residual.p)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                r.fit(k, exact, u[k]);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[k][j] += u[k][j];
            }
        float q = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) q += s[k][j] * s[k][j];             // channels behind the last are zeros
        const float rstd = inverse_root(total(q) / (float)a.c + a.eps);
#pragma unroll
        for (int k = 0; k < K; ++k) put_row(r, a, row0, k, exact, rstd, s[k]);
        if (r.lane == 0 && a.rstd) a.rstd[row] = rstd;
    }
}

// Rows too long for the registers of a workgroup: read twice.
template <int DT> __global__ __launch_bounds__(1024) void rms_long_rows_kernel(RmsArgs a)
{
    __shared__ float part[32];
    RowSum<1024> total{part};
    const Row<DT, 1024> r(a.c);
    const int K = (a.c + 8191) / 8192;
    for (long row = blockIdx.x; row < a.n; row += gridDim.x) {
        float s[8];
        auto values = [&](int k) {
            Words<DT, 8> x, u;
            r.load(r.from(a.x, row), 0, k, x);
            if (a.residual.p) r.load(r.from(a.residual, row), 0, k, u);
            r.fit(k, false, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] = x[j];
            if (a.residual.p) {
                r.fit(k, false, u);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] += u[j];
            }
        };
        float q = 0.f;
        for (int k = 0; k < K; ++k) {
            values(k);
            float t = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) t += s[j] * s[j];
            q += t;
        }
        const float rstd = inverse_root(total(q) / (float)a.c + a.eps);
        for (int k = 0; k < K; ++k) {
            values(k);
            put_row(r, a, row, k, false, rstd, s);
        }
        if (threadIdx.x == 0 && a.rstd) a.rstd[row] = rstd;
    }
}

// Eight channels of what was normalised, as a tensor holds them or in 8 bits; kept as they were read.
template <int DT, int G, bool HELD> struct Normed;
template <int DT, int G> struct Normed<DT, G, false> {
    Words<DT, 8> w;
    // row0: the first of the wave's, or ALONE: this lane's own
    template <bool ALONE> __device__ __forceinline__ void load(const Row<DT, G> &r, const RmsBwdArgs &a, long row0, int k)
    {
        r.load(r.from(a.s, row0), ALONE ? 0 : r.offset(a.s), k, w);
    }
    __device__ __forceinline__ void fit(const Row<DT, G> &r, int k, bool exact) { r.fit(k, exact, w); }
    __device__ __forceinline__ void forget() { w.forget(); }
    __device__ __forceinline__ void values(const RmsBwdArgs &, float (&f)[8]) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = w[j];
    }
};
template <int DT, int G> struct Normed<DT, G, true> {
    uint32_t c[2], byte;
    template <bool ALONE> __device__ __forceinline__ void load(const Row<DT, G> &r, const RmsBwdArgs &a, long row0, int k)
    {
        const int c0 = r.channel(k), left = r.c - c0;
        const PackedView &v = a.s8;
        const uint32_t row = ALONE || G >= 64 ? 0 : r.sub;
        load_codes(v.codes + row0 * v.sn + (row * (uint32_t)v.sn + (uint32_t)c0), left, c);
        byte = left > 0 ? v.scales[row0 * v.ssn + (row * (uint32_t)v.ssn + (uint32_t)c0 / 32)] : 127;
    }
    __device__ __forceinline__ void fit(const Row<DT, G> &, int, bool) {}
    __device__ __forceinline__ void forget() { asm volatile("" : "+v"(c[0]), "+v"(c[1])); }
    __device__ __forceinline__ void values(const RmsBwdArgs &a, float (&f)[8]) const { held_octet(a.s8, c, byte, f); }
};

// sums of channels c0 .. c0 + 7 of c
__device__ __forceinline__ void put_sums(float *out, int c, int c0, const float (&f)[8])
{
    if (c0 + 8 <= c) {
        *reinterpret_cast<line_t<0, 8> *>(out + c0) = packed<0, 8>(f);
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (c0 + j < c) out[c0 + j] = f[j];
    }
}

// dgamma of 64 channels over all rows, by one workgroup: eight lanes an octet each, eight rows a wave
template <int DT, int T, bool HELD> __device__ void rms_rows_sums(const RmsBwdArgs &a, int block)
{
    constexpr int W = T / 64;
    __shared__ float sums[W][64];
    const Row<DT, 8> r(a.c);
    const int wave = uniform(threadIdx.x >> 6);
    float dg[8] = {};
    for (long row0 = 8 * wave; row0 < a.n; row0 += 8 * W) {
        const long row = row0 + r.sub;
        if (row >= a.n) break;
        Words<DT, 8> vy;
        Normed<DT, 8, HELD> vs;
        r.load(r.from(a.dy, row), 0, block, vy);                // (64 bits: the rows may be far apart)
        vs.template load<true>(r, a, row, block);
        const float rstd = a.rstd[row];
        r.fit(block, false, vy);
        vs.fit(r, block, false);
        float s[8];
        vs.values(a, s);
#pragma unroll
        for (int j = 0; j < 8; ++j) dg[j] += vy[j] * (s[j] * rstd);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float g = sum_over_groups<8>(dg[j]);
        if ((threadIdx.x & 63) < 8) sums[wave][8 * r.lane + j] = g;
    }
    __syncthreads();
    const int c = block * 64 + threadIdx.x;
    if (threadIdx.x >= 64 || c >= a.c) return;
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) v += sums[i][threadIdx.x];
    a.dgamma[c] = v;
}

// Backwards: a workgroup takes R = T / G rows at a time, gridDim.x * R apart, and keeps its lanes' sums for dgamma in registers until the end, where they are added
// up over the R rows' lanes through LDS and go to the workgroup's copy of the scratch, or to dgamma itself if there is one workgroup.  16384 x 4096 bf16 from a
// sum in e4m3, with dsum: 472 MB in 89 us = 5.3 TB/s, and the copies' sum 4.8.
//
// ROLES, for few rows: the first `walkers` workgroups leave the sums alone, and each of the others takes them for 64 channels over all rows, which are read twice
// (from the L2): one launch and no workspace.
template <int DT, int G, int K, int T, bool HELD, bool ROLES> __global__ __launch_bounds__(T, 4) void rms_rows_bwd_kernel(RmsBwdArgs a, int walkers)
{
    if (ROLES && blockIdx.x >= (unsigned)walkers) {
        rms_rows_sums<DT, T, HELD>(a, blockIdx.x - walkers);
        return;
    }
    constexpr int W = T / 64, R = T / G;
    constexpr int each = G < 64 ? 1 : G / 64;           // waves that hold one row's channels
    __shared__ float part[G > 64 ? 2 * W : 1];
    __shared__ float sums[R > 1 && !ROLES ? W / each : 1][R > 1 && !ROLES ? G * K * 8 + 1 : 1];
    const Row<DT, G> r(a.c);
    const bool exact = a.c == 8 * G * K;
    const int wave = uniform(threadIdx.x >> 6), group = wave / each;
    float gamma[K][8], dg[K][8];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        Words<0, 8> g;
        if (a.gamma) {
            r.load(reinterpret_cast<src_t>(a.gamma), 0, k, g);
            r.fit(k, exact, g);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            gamma[k][j] = a.gamma ? g[j] : 1.f;
            dg[k][j] = 0.f;
        }
    }
    int half = 0;
    for (long first = blockIdx.x * (long)R; first < a.n; first += walkers * (long)R) {     // (every thread alike)
        const long row0 = first + (G < 64 ? wave * (64 / G) : group);
        const bool mine = row0 + r.sub < a.n;
        if (G <= 64 && !mine) continue;                 // (G > 64: all come to the barrier)
        Words<DT, 8> vy[K], vd[K];
        Normed<DT, G, HELD> vs[K];
        float rstd = 0.f, sgh = 0.f;
        if (mine) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                r.load(r.from(a.dy, row0), r.offset(a.dy), k, vy[k]);
                vs[k].template load<false>(r, a, row0, k);
            }
            if (a.dsum.p)
#pragma unroll
                for (int k = 0; k < K; ++k) r.load(r.from(a.dsum, row0), r.offset(a.dsum), k, vd[k]);
            rstd = a.rstd[row0 + r.sub];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                r.fit(k, exact, vy[k]);                 // behind the last channel dy and s are zero
                vs[k].fit(r, k, exact);
                float s[8];
                vs[k].values(a, s);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float y = vy[k][j], h = s[j] * rstd;
                    sgh += y * gamma[k][j] * h;
                    if (!ROLES) dg[k][j] += y * h;
                }
            }
        }
        sgh = sum_lanes<(G < 64 ? G : 64)>(sgh);
        if (G > 64) {
            float *p = part + half * W;                 // two halves in turn: one barrier a row
            half ^= 1;
            if ((threadIdx.x & 63) == 0) p[wave] = sgh;
            __syncthreads();
            sgh = 0.f;
#pragma unroll
            for (int i = 0; i < each; ++i) sgh += p[group * each + i];
        }
        if (!mine || !a.dx.p) continue;
        const float mean = sgh / (float)a.c;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (r.channel(k) >= a.c) continue;
            vy[k].forget();
            vs[k].forget();
            float s[8], t[8];
            vs[k].values(a, s);
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = rstd * (vy[k][j] * gamma[k][j] - s[j] * rstd * mean);
            if (a.dsum.p) {
                r.fit(k, exact, vd[k]);
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] += vd[k][j];
            }
            put_line(r, a.dx, row0, k, t);
        }
    }
    if (ROLES || !a.dgamma) return;
    float *out = gridDim.x == 1 ? a.dgamma : a.scratch + blockIdx.x * rms_copy_floats(a.c);
    if (R == 1) {                                       // every channel belongs to one lane of the workgroup
#pragma unroll
        for (int k = 0; k < K; ++k) put_sums(out, a.c, r.channel(k), dg[k]);
        return;
    }
    // rows of one wave first, then the groups in order
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float v = dg[k][j];
#pragma unroll
            for (int i = G; i < 64; i *= 2) v += __shfl_xor(v, i);
            if (G >= 64 || (threadIdx.x & 63) < G) sums[ROLES ? 0 : group][ROLES ? 0 : r.channel(k) + j] = v;
        }
    __syncthreads();
    for (int c = threadIdx.x; c < a.c; c += T) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < W / each; ++i) v += sums[ROLES ? 0 : i][ROLES ? 0 : c];
        out[c] = v;
    }
}

// Rows too long for the registers: read twice; dgamma by a walk over the rows per channel.
template <int DT, bool HELD> __global__ __launch_bounds__(1024) void rms_long_rows_bwd_kernel(RmsBwdArgs a)
{
    __shared__ float part[32];
    RowSum<1024> total{part};
    const Row<DT, 1024> r(a.c);
    const int K = (a.c + 8191) / 8192;
    for (long row = blockIdx.x; row < a.n; row += gridDim.x) {
        const float rstd = a.rstd[row];
        float s[8], g[8];
        auto both = [&](int k) {
            Words<DT, 8> vy;
            Normed<DT, 1024, HELD> vs;
            r.load(r.from(a.dy, row), 0, k, vy);
            vs.template load<false>(r, a, row, k);
            r.fit(k, false, vy);
            vs.fit(r, k, false);
            vs.values(a, s);
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = vy[j] * (a.gamma && r.channel(k) + j < a.c ? a.gamma[r.channel(k) + j] : 1.f);
        };
        float sgh = 0.f;
        for (int k = 0; k < K; ++k) {
            both(k);
            float t = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) t += g[j] * (s[j] * rstd);
            sgh += t;
        }
        const float mean = total(sgh) / (float)a.c;
        for (int k = 0; k < K; ++k) {
            both(k);
            if (r.channel(k) >= a.c) continue;
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = rstd * (g[j] - s[j] * rstd * mean);
            if (a.dsum.p) {
                Words<DT, 8> vd;
                r.load(r.from(a.dsum, row), 0, k, vd);
                r.fit(k, false, vd);
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] += vd[j];
            }
            put_line(r, a.dx, row, k, g);
        }
    }
}

// dgamma of rows too long for registers: a thread eight channels, blockIdx.y a share of the rows.  At most sixteen shares, few workgroups: 8192 x 16392 bf16 365 us of the gradient's
// 932 (rows of 16384, which fit: 155 in all).
template <int DT, bool HELD> __global__ __launch_bounds__(1024) void rms_long_rows_dgamma_kernel(RmsBwdArgs a)
{
    const Row<DT, 1024> r(a.c);
    for (int k = blockIdx.x; k < (a.c + 8191) / 8192; k += gridDim.x) {
        float dg[8] = {};
        for (long row = blockIdx.y; row < a.n; row += gridDim.y) {
            Words<DT, 8> vy;
            Normed<DT, 1024, HELD> vs;
            r.load(r.from(a.dy, row), 0, k, vy);
            vs.template load<false>(r, a, row, k);
            const float rstd = a.rstd[row];
            r.fit(k, false, vy);
            vs.fit(r, k, false);
            float s[8];
            vs.values(a, s);
#pragma unroll
            for (int j = 0; j < 8; ++j) dg[j] += vy[j] * (s[j] * rstd);
        }
        put_sums(gridDim.y == 1 ? a.dgamma : a.scratch + blockIdx.y * rms_copy_floats(a.c), a.c, r.channel(k), dg);
    }
}

constexpr int kLongRow = 32768, kLongRowBwd = 16384;    // longer rows do not fit the registers of a workgroup

// f(G, K, T) for rows of c channels, forwards; far: rows so far apart that 32 bits do not span those of a wave
template <class F> void pick_rows(int c, bool far, F f)
{
    if (c <= 8 && !far) return f(num<1>{}, num<1>{}, num<256>{});
    if (c <= 64 && !far) return f(num<8>{}, num<1>{}, num<256>{});
    if (c <= 256 && !far) return f(num<32>{}, num<1>{}, num<256>{});
    if (c <= 512) return f(num<64>{}, num<1>{}, num<256>{});
    if (c <= 1024) return f(num<64>{}, num<2>{}, num<256>{});
    if (c <= 2048) return f(num<64>{}, num<4>{}, num<256>{});
    if (c <= 4096) return f(num<256>{}, num<2>{}, num<256>{});
    if (c <= 8192) return f(num<256>{}, num<4>{}, num<256>{});
    if (c <= 16384) return f(num<1024>{}, num<2>{}, num<1024>{});
    return f(num<1024>{}, num<4>{}, num<1024>{});
}

// the same backwards, where a lane also holds gamma and a sum a channel
template <class F> void pick_rows_bwd(int c, bool far, F f)
{
    if (c <= 8 && !far) return f(num<1>{}, num<1>{}, num<512>{});
    if (c <= 64 && !far) return f(num<8>{}, num<1>{}, num<512>{});
    if (c <= 256 && !far) return f(num<32>{}, num<1>{}, num<512>{});
    if (c <= 512) return f(num<64>{}, num<1>{}, num<512>{});
    if (c <= 1024) return f(num<64>{}, num<2>{}, num<512>{});
    if (c <= 2048) return f(num<128>{}, num<2>{}, num<512>{});
    if (c <= 4096) return f(num<256>{}, num<2>{}, num<512>{});
    if (c <= 8192) return f(num<512>{}, num<2>{}, num<512>{});
    return f(num<1024>{}, num<2>{}, num<1024>{});
}

bool far_packed(std::initializer_list<const PackedView *> views)
{
    for (const PackedView *v : views)
        if (v->codes && (v->sn >= (1L << 24) || v->ssn >= (1L << 24))) return true;
    return false;
}

// Sixteen columns a workgroup: four lanes take a float4 each and 64 groups of them share the copies out, eight loads in flight.
__global__ __launch_bounds__(256) void rms_reduce_kernel(const float *scratch, int copies, float *dgamma, int c)
{
    typedef float floatx4 __attribute__((ext_vector_type(4)));
    __shared__ floatx4 sh[4][4];
    const int cp = (c + 3) / 4 * 4, group = threadIdx.x >> 2;
    for (int first = blockIdx.x * 16; first < cp; first += gridDim.x * 16) {        // (every thread alike)
        const int e = first + 4 * (threadIdx.x & 3);
        floatx4 s{};
        if (e < cp) {
            const float *p = scratch + e;
            int i = group;
            for (; i + 7 * 64 < copies; i += 8 * 64) {
                floatx4 v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] = *reinterpret_cast<const floatx4 *>(p + (long)(i + 64 * u) * cp);
                s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
            }
            for (; i < copies; i += 64) s += *reinterpret_cast<const floatx4 *>(p + (long)i * cp);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = sum_over_groups<4>(s[j]);
        if ((threadIdx.x & 63) < 4) sh[threadIdx.x >> 6][threadIdx.x & 3] = s;
        __syncthreads();
        if (threadIdx.x < 4 && e < cp) {
            s = (sh[0][threadIdx.x] + sh[1][threadIdx.x]) + (sh[2][threadIdx.x] + sh[3][threadIdx.x]);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (e + j < c) dgamma[e + j] = s[j];
        }
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_rms_reduce(const float *scratch, int copies, float *dgamma, int c, hipStream_t stream)
{
    rms_reduce_kernel<<<norm_blocks(rms_copy_floats(c), 16), 256, 0, stream>>>(scratch, copies, dgamma, c);
    return hipGetLastError();
}

hipError_t launch_rms_rows(const RmsArgs &a, hipStream_t stream)
{
    const bool far = far_apart({&a.x, &a.residual, &a.sum, &a.y}) || far_packed({&a.sum8, &a.y8});
    pick_dtype(a.dtype, [&](auto dt) {
        if (a.c > kLongRow) {
            rms_long_rows_kernel<dt()><<<norm_blocks(a.n, 1), 1024, 0, stream>>>(a);
            return;
        }
        pick_rows(a.c, far, [&](auto g, auto k, auto t) { rms_rows_kernel<dt(), g(), k(), t()><<<norm_blocks(a.n, t() / g()), t(), 0, stream>>>(a); });
    });
    return hipGetLastError();
}

// Where ROLES take the work: up to 512 rows, 1024 of more than 2048 channels.  With roles and with copies and a second launch, us, bf16 (fp32): 37 x 777 4.2 and 7.0 (3.8 and 6.8),
// 512 x 777 6.3 and 7.4 (7.2 and 7.2), 768 x 777 7.9 and 7.7 (10.6 and 7.6); 512 x 2048 4.7 and 7.6 (6.7 and 8.2), 1024 x 2048 10.0 and 9.2 (14 and 12); 512 x 4096 7.1 and 10.8 (10.8 and
// 13.9), 1024 x 4096 12.7 and 17.0 (17.8 and 17.0), 2048 x 4096 23 and 17 (30 and 24).
static bool takes_roles(const NormSpan &s) { return s.c > 8 && s.c <= kLongRowBwd && s.n <= (s.c > 2048 ? 1024 : 512); }

int rms_rows_bwd_copies(const NormSpan &s)
{
    if (s.c > kLongRowBwd) return (int)std::min<long>(s.n, 16);
    int copies = 1;
    if (takes_roles(s)) return copies;
    pick_rows_bwd(s.c, false, [&](auto g, auto, auto t) {
        const long rounds = (s.n + t() / g() - 1) / (t() / g());
        copies = rounds <= 4 && s.c <= 8 ? 1 : (int)std::min<long>(rounds, 256 * 1024 / t());       // (rows of up to eight channels have no roles)
    });
    return copies;
}

hipError_t launch_rms_rows_bwd(const RmsBwdArgs &a, hipStream_t stream)
{
    const int copies = rms_rows_bwd_copies(a);
    const bool in_place = a.dx.p && (a.dx.p == a.dy.p || a.dx.p == a.s.p);
    const bool far = far_apart({&a.dy, &a.s, &a.dsum, &a.dx}) || far_packed({&a.s8});
    Launches done;
    auto go = [&](auto dt, auto held) {
        if (a.c > kLongRowBwd) {
            if (a.dgamma) {
                rms_long_rows_dgamma_kernel<dt(), held()><<<dim3((unsigned)std::min((a.c + 8191) / 8192, 65536), copies), 1024, 0, stream>>>(a);
                if (done.failed() || (copies > 1 && done.failed(launch_rms_reduce(a.scratch, copies, a.dgamma, a.c, stream)))) return;
            }
            if (a.dx.p) rms_long_rows_bwd_kernel<dt(), held()><<<norm_blocks(a.n, 1), 1024, 0, stream>>>(a);
            return;
        }
        pick_rows_bwd(a.c, far, [&](auto g, auto k, auto t) {
            const long rounds = (a.n + t() / g() - 1) / (t() / g());
            const int all = (int)std::min<long>(rounds, 256 * 1024 / t());
            const bool roles = a.dgamma && takes_roles(a);
            if (roles) {
                const int walkers = a.dx.p && !in_place ? all : 0, blocks = walkers + (a.c + 63) / 64;
                rms_rows_bwd_kernel<dt(), g(), k(), t(), held(), true><<<blocks, t(), 0, stream>>>(a, walkers);
                if (done.failed() || walkers || !a.dx.p) return;
            }
            RmsBwdArgs b = a;
            if (roles) b.dgamma = nullptr;
            const int blocks = b.dgamma ? copies : all;
            rms_rows_bwd_kernel<dt(), g(), k(), t(), held(), false><<<blocks, t(), 0, stream>>>(b, blocks);
            if (!done.failed() && b.dgamma && blocks > 1) done.failed(launch_rms_reduce(a.scratch, blocks, a.dgamma, a.c, stream));
        });
    };
    pick_dtype(a.dtype, [&](auto dt) {
        if (a.s8.codes) go(dt, std::true_type{});
        else go(dt, std::false_type{});
    });
    return done.status();
}

}  // namespace sk
