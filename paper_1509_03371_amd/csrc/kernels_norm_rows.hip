// Layer norm of rows: the channels of a position side by side.
#include "norm_device.h"
#include "reduce_copies.h"

namespace sk {

namespace {

// A row belongs to G lanes; lane l holds channels 8*(k*G + l) .. + 7 for k < K, the whole row in registers: one read of every input, one write of
// every output, and the variance from the values themselves about their mean.  T threads a workgroup; G > 64: G = T, sums through LDS.
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

template <int DT, int G, int K, int T> __global__ __launch_bounds__(T) void norm_rows_kernel(NormArgs a)
{
    typedef elem_t<DT> E;
    __shared__ float part[G > 64 ? 2 * (G / 64) : 1];
    RowSum<G> total{part};
    const int lane = threadIdx.x % G;
    const uint64_t base = a.drop.base();
    for (long row = blockIdx.x * (long)(T / G) + threadIdx.x / G; row < a.n; row += gridDim.x * (long)(T / G)) {     // (G > 64: every thread alike)
        const E *x = static_cast<const E *>(a.x.p) + row * a.x.sn;
        float s[K][8];
        {
            line_t<DT, 8> v[K];
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] = load_line<DT, 8>(x, 8 * (k * G + lane), a.c);
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) s[k][j] = (float)v[k][j];
        }
        if (a.drop.thresh) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                uint32_t w[4];
                mask_words(w, a.drop, base, (uint64_t)row, k * G + lane);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[k][j] = dropped(s[k][j], w, j, a.drop);
            }
        }
        if (a.residual.p) {
            const E *r = static_cast<const E *>(a.residual.p) + row * a.residual.sn;
            line_t<DT, 8> v[K];
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] = load_line<DT, 8>(r, 8 * (k * G + lane), a.c);
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) s[k][j] += (float)v[k][j];
        }
        float sum = 0.f, var = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += s[k][j];     // channels beyond the last are zeros
        const float mean = total(sum) / (float)a.c;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = 8 * (k * G + lane) + j < a.c ? s[k][j] - mean : 0.f;
                var += d * d;
            }
        const float rstd = 1.f / sqrtf(total(var) / (float)a.c + a.eps);
        E *y = static_cast<E *>(a.y.p) + row * a.y.sn;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c0 = 8 * (k * G + lane);
            if (c0 >= a.c) break;
            if (a.sum.p) store_line<DT, 8>(static_cast<E *>(a.sum.p) + row * a.sum.sn, c0, a.c, s[k]);
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = (s[k][j] - mean) * rstd;
            if (a.gamma) {
                const line_t<0, 8> g = load_line<0, 8>(a.gamma, c0, a.c);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] *= g[j];
            }
            if (a.beta) {
                const line_t<0, 8> b = load_line<0, 8>(a.beta, c0, a.c);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] += b[j];
            }
            if (a.relu)
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = o[j] < 0.f ? 0.f : o[j];
            store_line<DT, 8>(y, c0, a.c, o);
        }
        if (lane == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// Rows too long for the registers of a workgroup: read three times.
template <int DT> __global__ __launch_bounds__(1024) void norm_long_rows_kernel(NormArgs a)
{
    typedef elem_t<DT> E;
    __shared__ float part[32];
    RowSum<1024> total{part};
    for (long row = blockIdx.x; row < a.n; row += gridDim.x) {
        const E *x = static_cast<const E *>(a.x.p) + row * a.x.sn, *r = static_cast<const E *>(a.residual.p) + row * a.residual.sn;
        const uint64_t base = a.drop.base();
        auto values = [&](int c0, float (&s)[8]) {
            const line_t<DT, 8> v = load_line<DT, 8>(x, c0, a.c);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] = (float)v[j];
            if (a.drop.thresh) {
                uint32_t w[4];
                mask_words(w, a.drop, base, (uint64_t)row, (uint32_t)c0 >> 3);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] = dropped(s[j], w, j, a.drop);
            }
            if (a.residual.p) {
                const line_t<DT, 8> u = load_line<DT, 8>(r, c0, a.c);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] += (float)u[j];
            }
        };
        float sum = 0.f, var = 0.f, s[8];
        for (int c0 = 8 * threadIdx.x; c0 < a.c; c0 += 8192) {
            values(c0, s);
            float t = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) t += s[j];
            sum += t;
        }
        const float mean = total(sum) / (float)a.c;
        for (int c0 = 8 * threadIdx.x; c0 < a.c; c0 += 8192) {
            values(c0, s);
            float t = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = c0 + j < a.c ? s[j] - mean : 0.f;
                t += d * d;
            }
            var += t;
        }
        const float rstd = 1.f / sqrtf(total(var) / (float)a.c + a.eps);
        for (int c0 = 8 * threadIdx.x; c0 < a.c; c0 += 8192) {
            values(c0, s);
            if (a.sum.p) store_line<DT, 8>(static_cast<E *>(a.sum.p) + row * a.sum.sn, c0, a.c, s);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float o = (s[j] - mean) * rstd;
                if (c0 + j < a.c) {
                    if (a.gamma) o *= a.gamma[c0 + j];
                    if (a.beta) o += a.beta[c0 + j];
                }
                s[j] = a.relu && o < 0.f ? 0.f : o;
            }
            store_line<DT, 8>(static_cast<E *>(a.y.p) + row * a.y.sn, c0, a.c, s);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// Backwards: a workgroup walks rows gridDim.x * T / G apart and keeps its lanes' sums for dgamma and dbeta in registers until the end, where they
// go to the workgroup's copy [2][c rounded up to 4] of the scratch, or to dgamma and dbeta themselves if there is one workgroup.
template <int DT, int G, int K, int T> __global__ __launch_bounds__(T) void norm_rows_bwd_kernel(NormBwdArgs a)
{
    typedef elem_t<DT> E;
    constexpr int R = T / G;                            // rows at a time
    constexpr int W = T / 64;
    __shared__ float part[G > 64 ? 4 * W : 1];
    __shared__ float sums[G < T ? W : 1][G < T ? 64 * K * 8 + 1 : 1];
    const int lane = threadIdx.x % G;
    const uint64_t base = a.drop.base();
    float gamma[K][8], dg[K][8], db[K][8];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c0 = 8 * (k * G + lane);
        const line_t<0, 8> g = a.gamma ? load_line<0, 8>(a.gamma, c0, a.c) : line_t<0, 8>{};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            gamma[k][j] = a.gamma ? g[j] : c0 + j < a.c ? 1.f : 0.f;
            dg[k][j] = db[k][j] = 0.f;
        }
    }
    int half = 0;
    for (long row = blockIdx.x * (long)R + threadIdx.x / G; row < a.n; row += gridDim.x * (long)R) {     // (G > 64: R = 1, every thread alike)
        const E *dy = static_cast<const E *>(a.dy.p) + row * a.dy.sn, *s = static_cast<const E *>(a.s.p) + row * a.s.sn;
        line_t<DT, 8> vy[K], vs[K], vd[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            vy[k] = load_line<DT, 8>(dy, 8 * (k * G + lane), a.c);
            vs[k] = load_line<DT, 8>(s, 8 * (k * G + lane), a.c);
        }
        if (a.dsum.p)
#pragma unroll
            for (int k = 0; k < K; ++k) vd[k] = load_line<DT, 8>(static_cast<const E *>(a.dsum.p) + row * a.dsum.sn, 8 * (k * G + lane), a.c);
        const float mean = a.mean[row], rstd = a.rstd[row];
        float sg = 0.f, sgh = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float h = ((float)vs[k][j] - mean) * rstd, y = (float)vy[k][j], g = y * gamma[k][j];     // beyond the last channel y is zero
                sg += g;
                sgh += g * h;
                dg[k][j] += y * h;
                db[k][j] += y;
            }
        sg = sum_lanes<(G < 64 ? G : 64)>(sg);
        sgh = sum_lanes<(G < 64 ? G : 64)>(sgh);
        if (G > 64) {
            float *p = part + half * 2 * W;             // two halves in turn: one barrier a row
            half ^= 1;
            if ((threadIdx.x & 63) == 0) {
                p[threadIdx.x >> 6] = sg;
                p[W + (threadIdx.x >> 6)] = sgh;
            }
            __syncthreads();
            sg = sgh = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                sg += p[i];
                sgh += p[W + i];
            }
        }
        if (!a.dx.p && !a.dresidual.p) continue;
        const float mg = sg / (float)a.c, mgh = sgh / (float)a.c;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c0 = 8 * (k * G + lane);
            if (c0 >= a.c) break;
            float t[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float h = ((float)vs[k][j] - mean) * rstd;
                t[j] = rstd * ((float)vy[k][j] * gamma[k][j] - mg - h * mgh);
            }
            if (a.dsum.p)
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] += (float)vd[k][j];
            if (a.dresidual.p) store_line<DT, 8>(static_cast<E *>(a.dresidual.p) + row * a.dresidual.sn, c0, a.c, t);
            if (!a.dx.p) continue;
            if (a.drop.thresh) {
                uint32_t w[4];
                mask_words(w, a.drop, base, (uint64_t)row, k * G + lane);
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] = dropped(t[j], w, j, a.drop);
            }
            if (a.relu_x)
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] = (float)vs[k][j] > 0.f ? t[j] : 0.f;
            store_line<DT, 8>(static_cast<E *>(a.dx.p) + row * a.dx.sn, c0, a.c, t);
        }
    }
    if (!a.dgamma && !a.dbeta) return;
    const bool alone = gridDim.x == 1;
    const long cp = norm_copy_floats(a.c) / 2;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float(&acc)[K][8] = which ? db : dg;
        float *out = alone ? (which ? a.dbeta : a.dgamma) : a.scratch + (blockIdx.x * 2L + which) * cp;
        const long count = alone ? a.c : cp;            // a copy's tail holds zeros
        if (G == T) {                                   // every channel belongs to one lane of the workgroup
            if (out)
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const int c0 = 8 * (k * G + lane);
                    if (c0 < count) store_line<0, 8>(out, c0, count, acc[k]);
                }
            continue;
        }
        // rows of one wave first, then the waves in order
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float v = acc[k][j];
#pragma unroll
                for (int i = G; i < 64; i *= 2) v += __shfl_xor(v, i);
                if ((threadIdx.x & 63) < G) sums[threadIdx.x >> 6][8 * (k * G + lane) + j] = v;
            }
        __syncthreads();
        if (out)
            for (int c = threadIdx.x; c < count; c += T) {
                float v = 0.f;
                if (c < 8 * K * G)
#pragma unroll
                    for (int i = 0; i < W; ++i) v += sums[i][c];
                out[c] = v;
            }
        __syncthreads();
    }
}

// Rows too long for the registers: read twice; the sums of dgamma and dbeta by a walk over the rows per channel.
template <int DT> __global__ __launch_bounds__(1024) void norm_long_rows_bwd_kernel(NormBwdArgs a)
{
    typedef elem_t<DT> E;
    __shared__ float part[32];
    RowSum<1024> total{part};
    for (long row = blockIdx.x; row < a.n; row += gridDim.x) {
        const E *dy = static_cast<const E *>(a.dy.p) + row * a.dy.sn, *s = static_cast<const E *>(a.s.p) + row * a.s.sn;
        const uint64_t base = a.drop.base();
        const float mean = a.mean[row], rstd = a.rstd[row];
        float sg = 0.f, sgh = 0.f;
        auto both = [&](int c0, float (&g)[8], float (&v)[8]) {
            const line_t<DT, 8> vy = load_line<DT, 8>(dy, c0, a.c), vs = load_line<DT, 8>(s, c0, a.c);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = (float)vs[j];
                g[j] = (float)vy[j] * (a.gamma && c0 + j < a.c ? a.gamma[c0 + j] : 1.f);
            }
        };
        float g[8], v[8];
        for (int c0 = 8 * threadIdx.x; c0 < a.c; c0 += 8192) {
            both(c0, g, v);
            float t0 = 0.f, t1 = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                t0 += g[j];
                t1 += g[j] * ((v[j] - mean) * rstd);
            }
            sg += t0;
            sgh += t1;
        }
        const float mg = total(sg) / (float)a.c, mgh = total(sgh) / (float)a.c;
        for (int c0 = 8 * threadIdx.x; c0 < a.c; c0 += 8192) {
            both(c0, g, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = rstd * (g[j] - mg - (v[j] - mean) * rstd * mgh);
            if (a.dsum.p) {
                const line_t<DT, 8> d = load_line<DT, 8>(static_cast<const E *>(a.dsum.p) + row * a.dsum.sn, c0, a.c);
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] += (float)d[j];
            }
            if (a.dresidual.p) store_line<DT, 8>(static_cast<E *>(a.dresidual.p) + row * a.dresidual.sn, c0, a.c, g);
            if (!a.dx.p) continue;
            if (a.drop.thresh) {
                uint32_t w[4];
                mask_words(w, a.drop, base, (uint64_t)row, (uint32_t)c0 >> 3);
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] = dropped(g[j], w, j, a.drop);
            }
            if (a.relu_x)
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] = v[j] > 0.f ? g[j] : 0.f;
            store_line<DT, 8>(static_cast<E *>(a.dx.p) + row * a.dx.sn, c0, a.c, g);
        }
    }
}

// dgamma and dbeta of rows too long for registers: a thread eight channels, blockIdx.y a share of the rows
template <int DT> __global__ __launch_bounds__(256) void norm_long_rows_wgrad_kernel(NormBwdArgs a)
{
    typedef elem_t<DT> E;
    const int c0 = 8 * (blockIdx.x * 256 + threadIdx.x);
    const long cp = norm_copy_floats(a.c) / 2;
    if (c0 >= cp) return;
    float dg[8] = {}, db[8] = {};
    for (long row = blockIdx.y; row < a.n; row += gridDim.y) {
        const line_t<DT, 8> vy = load_line<DT, 8>(static_cast<const E *>(a.dy.p) + row * a.dy.sn, c0, a.c);
        const line_t<DT, 8> vs = load_line<DT, 8>(static_cast<const E *>(a.s.p) + row * a.s.sn, c0, a.c);
        const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            dg[j] += (float)vy[j] * (((float)vs[j] - mean) * rstd);
            db[j] += (float)vy[j];
        }
    }
    float *out = a.scratch + blockIdx.y * 2L * cp;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (c0 + j < cp) {
            out[c0 + j] = c0 + j < a.c ? dg[j] : 0.f;
            out[cp + c0 + j] = c0 + j < a.c ? db[j] : 0.f;
        }
}

constexpr int kLongRow = 32768;                         // from here on rows do not fit the registers of a workgroup

// f(G, K, T) for rows of c channels, forwards
template <class F> hipError_t pick_rows(int c, F f)
{
#define SK_ROWS_CASE(most, G, K, T) if (c <= most) return f(std::integral_constant<int, G>{}, std::integral_constant<int, K>{}, std::integral_constant<int, T>{})
    SK_ROWS_CASE(8, 1, 1, 256);
    SK_ROWS_CASE(64, 8, 1, 256);
    SK_ROWS_CASE(128, 16, 1, 256);
    SK_ROWS_CASE(256, 32, 1, 256);
    SK_ROWS_CASE(512, 64, 1, 256);
    SK_ROWS_CASE(1024, 64, 2, 256);
    SK_ROWS_CASE(2048, 64, 4, 256);
    SK_ROWS_CASE(4096, 256, 2, 256);
    SK_ROWS_CASE(8192, 256, 4, 256);
    SK_ROWS_CASE(16384, 1024, 2, 1024);
    return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 4>{}, std::integral_constant<int, 1024>{});
}

// the same backwards, where a lane also holds gamma and two sums a channel
template <class F> hipError_t pick_rows_bwd(int c, F f)
{
    SK_ROWS_CASE(8, 1, 1, 256);
    SK_ROWS_CASE(64, 8, 1, 256);
    SK_ROWS_CASE(128, 16, 1, 256);
    SK_ROWS_CASE(256, 32, 1, 256);
    SK_ROWS_CASE(512, 64, 1, 256);
    SK_ROWS_CASE(1024, 64, 2, 256);
    SK_ROWS_CASE(2048, 128, 2, 128);
    SK_ROWS_CASE(4096, 256, 2, 256);
    SK_ROWS_CASE(8192, 512, 2, 512);
    SK_ROWS_CASE(16384, 1024, 2, 1024);
    return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 4>{}, std::integral_constant<int, 1024>{});
#undef SK_ROWS_CASE
}

template <class F> hipError_t pick_type(int dtype, F f)
{
    if (dtype == 0) return f(std::integral_constant<int, 0>{});
    if (dtype == 1) return f(std::integral_constant<int, 1>{});
    return f(std::integral_constant<int, 2>{});
}

__global__ __launch_bounds__(256) void norm_reduce_kernel(const float *scratch, int copies, float *dgamma, float *dbeta, int c)
{
    __shared__ float sh[16][64];
    const int cp = (c + 3) / 4 * 4, e = blockIdx.x * 64 + threadIdx.x;
    const float v = sum_copies64(scratch, 2L * cp, blockIdx.x * 64, 2 * cp, copies, sh);
    if (threadIdx.x >= 64 || e >= 2 * cp) return;
    float *out = e < cp ? dgamma : dbeta;
    const int k = e < cp ? e : e - cp;
    if (out && k < c) out[k] = v;
}

}  // namespace

hipError_t launch_norm_reduce(const float *scratch, int copies, float *dgamma, float *dbeta, int c, hipStream_t stream)
{
    norm_reduce_kernel<<<(unsigned)((norm_copy_floats(c) + 63) / 64), 256, 0, stream>>>(scratch, copies, dgamma, dbeta, c);
    return hipGetLastError();
}

hipError_t launch_norm_rows(const NormArgs &a, hipStream_t stream)
{
    return pick_type(a.dtype, [&](auto dt) {
        if (a.c > kLongRow) {
            norm_long_rows_kernel<dt()><<<norm_blocks(a.n, 1), 1024, 0, stream>>>(a);
            return hipGetLastError();
        }
        return pick_rows(a.c, [&](auto g, auto k, auto t) {
            norm_rows_kernel<dt(), g(), k(), t()><<<norm_blocks(a.n, t() / g()), t(), 0, stream>>>(a);
            return hipGetLastError();
        });
    });
}

int norm_rows_bwd_copies(const NormSpan &s)
{
    if (s.c > kLongRow) return (int)std::min<long>(s.n, 16);
    int copies = 1;
    (void)pick_rows_bwd(s.c, [&](auto g, auto, auto t) {
        copies = (int)std::min<long>((s.n + t() / g() - 1) / (t() / g()), 256 * 1024 / t());
        return hipSuccess;
    });
    return copies;
}

hipError_t launch_norm_rows_bwd(const NormBwdArgs &a, int copies, hipStream_t stream)
{
    return pick_type(a.dtype, [&](auto dt) {
        if (a.c > kLongRow) {
            if (a.dgamma || a.dbeta) {
                norm_long_rows_wgrad_kernel<dt()><<<dim3((unsigned)((a.c + 2047) / 2048), copies), 256, 0, stream>>>(a);
                if (hipError_t e = launch_norm_reduce(a.scratch, copies, a.dgamma, a.dbeta, a.c, stream)) return e;
            }
            if (a.dx.p || a.dresidual.p) norm_long_rows_bwd_kernel<dt()><<<norm_blocks(a.n, 1), 1024, 0, stream>>>(a);
            return hipGetLastError();
        }
        return pick_rows_bwd(a.c, [&](auto g, auto k, auto t) {
            norm_rows_bwd_kernel<dt(), g(), k(), t()><<<copies, t(), 0, stream>>>(a);
            if ((a.dgamma || a.dbeta) && copies > 1) return launch_norm_reduce(a.scratch, copies, a.dgamma, a.dbeta, a.c, stream);
            return hipGetLastError();
        });
    });
}

}  // namespace sk
