// Layer norm of rows: the channels of a position side by side.
#include "norm_row.h"

namespace sk {

namespace {

// HBM bounds the forward pass: 65536 x 2048 bf16 537 MB in 103.5 us = 5.2 TB/s, with residual, dropout and sum 16384 x 4096 bf16 537 MB in 94 us =
// 5.7 TB/s (copies of 512 MB: 5.1 to 5.3; under a trace 107 to 112 and 95); the first kernel, which read each row three times, took 544 and 605 us.

// ADD: what is normalised is residual + dropout(x), or is wanted as an output
template <int DT, int G, int K, int T, bool ADD> __global__ __launch_bounds__(T) void norm_rows_kernel(NormArgs a)
{
    __shared__ float part[G > 64 ? 2 * (G / 64) : 1];
    RowSum<G> total{part};
    const Row<DT, G> r(a.c);
    const bool exact = a.c == 8 * G * K;
    const uint64_t counter = ADD ? a.drop.base() : 0;
    for (long row0 = first_row<G, T>(); row0 < a.n; row0 += row_step<G, T>()) {     // (G > 64: every thread alike)
        const long row = row0 + r.sub;
        if (G < 64 && row >= a.n) break;
        float s[K][8];
        Words<DT, 8> x[K], u[ADD ? K : 1];
#pragma unroll
        for (int k = 0; k < K; ++k) r.load(r.from(a.x, row0), r.offset(a.x), k, x[k]);
        if (ADD && a.residual.p)
#pragma unroll
            for (int k = 0; k < K; ++k) r.load(r.from(a.residual, row0), r.offset(a.residual), k, u[ADD ? k : 0]);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            r.fit(k, exact, x[k]);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[k][j] = x[k][j];
        }
        if (ADD && a.drop.thresh)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                uint32_t w[4];
                mask_words(w, a.drop, counter, (uint64_t)row, k * G + r.lane);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[k][j] = dropped(s[k][j], w, j, a.drop);
            }
        if (ADD && a.residual.p)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                r.fit(k, exact, u[ADD ? k : 0]);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[k][j] += u[ADD ? k : 0][j];
            }
        float sum = 0.f, var = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += s[k][j];     // channels behind the last are zeros
        const float mean = total(sum) / (float)a.c;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = s[k][j] - mean;
                var += exact || r.channel(k) + j < a.c ? d * d : 0.f;
            }
        const float rstd = 1.f / sqrtf(total(var) / (float)a.c + a.eps);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (r.channel(k) >= a.c) continue;
            if (ADD && a.sum.p) r.store(a.sum, row0, k, s[k]);
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = (s[k][j] - mean) * rstd;
            if (a.gamma) {
                Words<0, 8> g;
                r.load(reinterpret_cast<src_t>(a.gamma), 0, k, g);
                r.fit(k, exact, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] *= g[j];
            }
            if (a.beta) {
                Words<0, 8> b;
                r.load(reinterpret_cast<src_t>(a.beta), 0, k, b);
                r.fit(k, exact, b);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] += b[j];
            }
            r.store(a.y, row0, k, o);
        }
        if (r.lane == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// Rows too long for the registers of a workgroup: read three times.
template <int DT> __global__ __launch_bounds__(1024) void norm_long_rows_kernel(NormArgs a)
{
    __shared__ float part[32];
    RowSum<1024> total{part};
    const Row<DT, 1024> r(a.c);
    const int K = (a.c + 8191) / 8192;
    const uint64_t counter = a.drop.base();
    for (long row = blockIdx.x; row < a.n; row += gridDim.x) {
        auto values = [&](int k, float (&s)[8]) {
            Words<DT, 8> x, u;
            r.load(r.from(a.x, row), 0, k, x);
            if (a.residual.p) r.load(r.from(a.residual, row), 0, k, u);
            r.fit(k, false, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] = x[j];
            if (a.drop.thresh) {
                uint32_t w[4];
                mask_words(w, a.drop, counter, (uint64_t)row, k * 1024 + r.lane);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] = dropped(s[j], w, j, a.drop);
            }
            if (a.residual.p) {
                r.fit(k, false, u);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] += u[j];
            }
        };
        float sum = 0.f, var = 0.f, s[8];
        for (int k = 0; k < K; ++k) {
            values(k, s);
            float t = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) t += s[j];
            sum += t;
        }
        const float mean = total(sum) / (float)a.c;
        for (int k = 0; k < K; ++k) {
            values(k, s);
            float t = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = s[j] - mean;
                t += r.channel(k) + j < a.c ? d * d : 0.f;
            }
            var += t;
        }
        const float rstd = 1.f / sqrtf(total(var) / (float)a.c + a.eps);
        for (int k = 0; k < K; ++k) {
            values(k, s);
            const int c0 = r.channel(k);
            if (c0 >= a.c) break;
            if (a.sum.p) r.store(a.sum, row, k, s);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s[j] = (s[j] - mean) * rstd;
                if (c0 + j < a.c) {
                    if (a.gamma) s[j] *= a.gamma[c0 + j];
                    if (a.beta) s[j] += a.beta[c0 + j];
                }
            }
            r.store(a.y, row, k, s);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// The gradient of a row's eight channels from its dy and s (kept as they were read) and the row's four numbers.  ADD: with dropout, dsum or dresidual.
template <bool ADD, int DT, int G>
__device__ __forceinline__ void put_gradients(const Row<DT, G> &r, const NormBwdArgs &a, uint64_t counter, long row0, int k, const Words<DT, 8> &vy,
                                              const Words<DT, 8> &vs, const Words<DT, 8> &vd, const float (&gamma)[8], float mean, float rstd, float mg,
                                              float mgh)
{
    const float mr = mgh * rstd;                        // rstd (gamma dy - mg - h mgh) with h = (s - mean) rstd
    float t[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) t[j] = rstd * (product(vy[j], gamma[j]) - mg - (vs[j] - mean) * mr);
    if (ADD) {
        if (a.dsum.p)
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] += vd[j];
        if (a.dresidual.p) r.store(a.dresidual, row0, k, t);
        if (!a.dx.p) return;
        if (a.drop.thresh) {
            uint32_t w[4];
            mask_words(w, a.drop, counter, (uint64_t)(row0 + r.sub), k * G + r.lane);
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = dropped(t[j], w, j, a.drop);
        }
    }
    r.store(a.dx, row0, k, t);
}

// sums of channels c0 .. c0 + 7 of c, which the reduction reads
__device__ __forceinline__ void put_values(float *out, int c, int c0, const float (&f)[8])
{
    if (c0 + 8 <= c) {
        *reinterpret_cast<line_t<0, 8> *>(out + c0) = packed<0, 8>(f);
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (c0 + j < c) out[c0 + j] = f[j];
    }
}

// Backwards: a workgroup takes R = T / G rows at a time, gridDim.x * R apart, and keeps its lanes' sums for dgamma and dbeta in registers until the end,
// where they are added up over the R rows' lanes through LDS and go to the workgroup's copy [2][c rounded up to 4] of the scratch, or to dgamma and dbeta
// themselves if there is one workgroup.  Eight waves a workgroup: with four, twice the copies, whose writing and adding up made 147 us of 134 for
// 16384 x 4096 bf16 with dropout and residual (671 MB: 5.1 TB/s).  Few rows a wave are bound by latency: 8192 x 1001 fp16, two rows a wave, 15 us for 49 MB.
// With residual or dropout 513 to 1024 channels spill registers (43 in fp32, 13 in 16 bits; wider fp32 rows 16 to 20): 16384 x 1024 fp32 336 MB in 83 us = 4.0
// TB/s, bf16 168 MB in 43 = 3.9.
//
// ROLES, for few rows: the first `walkers` workgroups leave the sums alone, and each of the others takes them for 64 channels over all rows, which are read twice
// (from the L2): one launch and no workspace.
template <int DT, int T> __device__ void norm_rows_sums(const NormBwdArgs &a, int block)
{
    constexpr int W = T / 64;
    __shared__ float sums[W][2][64];
    const Row<DT, 8> r(a.c);                            // eight lanes an octet each, eight rows a wave
    const int wave = uniform(threadIdx.x >> 6);
    const long to_dy = (long)r.S * r.sub * a.dy.sn, to_s = (long)r.S * r.sub * a.s.sn;     // 64 bits: the rows may be far apart
    float dg[8] = {}, db[8] = {};
    for (long row0 = 8 * wave; row0 < a.n; row0 += 8 * W) {
        if (row0 + r.sub >= a.n) break;
        Words<DT, 8> vy, vs;
        r.load(r.from(a.dy, row0) + to_dy, 0, block, vy);
        r.load(r.from(a.s, row0) + to_s, 0, block, vs);
        const float mean = a.mean[row0 + r.sub], rstd = a.rstd[row0 + r.sub];
        r.fit(block, false, vy);
        r.fit(block, false, vs);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            dg[j] += vy[j] * rstd * (vs[j] - mean);
            db[j] += vy[j];
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float g = sum_over_groups<8>(dg[j]), b = sum_over_groups<8>(db[j]);
        if ((threadIdx.x & 63) < 8) {
            sums[wave][0][8 * r.lane + j] = g;
            sums[wave][1][8 * r.lane + j] = b;
        }
    }
    __syncthreads();
    const int which = threadIdx.x >> 6, c = block * 64 + (threadIdx.x & 63);
    float *out = which ? a.dbeta : a.dgamma;
    if (which > 1 || c >= a.c || !out) return;
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) v += sums[i][which][threadIdx.x & 63];
    out[c] = v;
}

template <int DT, int G, int K, int T, bool ADD, bool ROLES> __global__ __launch_bounds__(T, 4) void norm_rows_bwd_kernel(NormBwdArgs a, int walkers)
{
    if (ROLES && blockIdx.x >= (unsigned)walkers) {
        norm_rows_sums<DT, T>(a, blockIdx.x - walkers);
        return;
    }
    constexpr int W = T / 64, R = T / G;
    constexpr int each = G < 64 ? 1 : G / 64;           // waves that hold one row's channels
    __shared__ float part[G > 64 ? 4 * W : 1];
    __shared__ float sums[R > 1 ? W / each : 1][R > 1 ? G * K * 8 + 1 : 1];
    const Row<DT, G> r(a.c);
    const bool exact = a.c == 8 * G * K;
    const uint64_t counter = ADD ? a.drop.base() : 0;
    const int wave = uniform(threadIdx.x >> 6), group = wave / each;
    float gamma[K][8], dg[K][8], db[K][8];
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
            dg[k][j] = db[k][j] = 0.f;
        }
    }
    int half = 0;
    for (long first = blockIdx.x * (long)R; first < a.n; first += walkers * (long)R) {     // (every thread alike)
        const long row0 = first + (G < 64 ? wave * (64 / G) : group);
        const bool mine = row0 + r.sub < a.n;
        if (G <= 64 && !mine) continue;                 // (G > 64: all come to the barrier)
        Words<DT, 8> vy[K], vs[K], vd[ADD ? K : 1];
        float mean = 0.f, rstd = 0.f, sg = 0.f, sgh = 0.f;
        if (mine) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                r.load(r.from(a.dy, row0), r.offset(a.dy), k, vy[k]);
                r.load(r.from(a.s, row0), r.offset(a.s), k, vs[k]);
            }
            if (ADD && a.dsum.p)
#pragma unroll
                for (int k = 0; k < K; ++k) r.load(r.from(a.dsum, row0), r.offset(a.dsum), k, vd[ADD ? k : 0]);
            mean = a.mean[row0 + r.sub];
            rstd = a.rstd[row0 + r.sub];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                r.fit(k, exact, vy[k]);                 // behind the last channel dy is zero
                r.fit(k, exact, vs[k]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float d = vs[k][j] - mean, y = vy[k][j], g = product(y, gamma[k][j]);
                    sg += g;
                    sgh += g * d;
                    if (ROLES) continue;
                    dg[k][j] += y * rstd * d;
                    db[k][j] += y;
                }
            }
            sgh *= rstd;
        }
        sg = sum_lanes<(G < 64 ? G : 64)>(sg);
        sgh = sum_lanes<(G < 64 ? G : 64)>(sgh);
        if (G > 64) {
            float *p = part + half * 2 * W;             // two halves in turn: one barrier a row
            half ^= 1;
            if ((threadIdx.x & 63) == 0) {
                p[wave] = sg;
                p[W + wave] = sgh;
            }
            __syncthreads();
            sg = sgh = 0.f;
#pragma unroll
            for (int i = 0; i < each; ++i) {
                sg += p[group * each + i];
                sgh += p[W + group * each + i];
            }
        }
        if (!mine || (!a.dx.p && (!ADD || !a.dresidual.p))) continue;
        const float mg = sg / (float)a.c, mgh = sgh / (float)a.c;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (r.channel(k) >= a.c) continue;
            if (ADD) {                                  // (where no registers are left for the values)
                vy[k].forget();
                vs[k].forget();
            }
            if (ADD && a.dsum.p) r.fit(k, exact, vd[ADD ? k : 0]);
            put_gradients<ADD>(r, a, counter, row0, k, vy[k], vs[k], vd[ADD ? k : 0], gamma[k], mean, rstd, mg, mgh);
        }
    }
    if (ROLES || (!a.dgamma && !a.dbeta)) return;
    const bool alone = gridDim.x == 1;
    const long cp = norm_copy_floats(a.c) / 2;
    auto put = [&](const float (&acc)[K][8], float *own, int which) {
        float *out = alone ? own : a.scratch + (blockIdx.x * 2L + which) * cp;
        if (R == 1) {                                   // every channel belongs to one lane of the workgroup
            if (out)
#pragma unroll
                for (int k = 0; k < K; ++k) put_values(out, a.c, r.channel(k), acc[k]);
            return;
        }
        // rows of one wave first, then the groups in order
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float v = acc[k][j];
#pragma unroll
                for (int i = G; i < 64; i *= 2) v += __shfl_xor(v, i);
                if (G >= 64 || (threadIdx.x & 63) < G) sums[group][r.channel(k) + j] = v;
            }
        __syncthreads();
        if (out)
            for (int c = threadIdx.x; c < a.c; c += T) {
                float v = 0.f;
#pragma unroll
                for (int i = 0; i < W / each; ++i) v += sums[i][c];
                out[c] = v;
            }
        __syncthreads();
    };
    put(dg, a.dgamma, 0);
    put(db, a.dbeta, 1);
}

// Rows too long for the registers: read twice; the sums of dgamma and dbeta by a walk over the rows per channel.
template <int DT> __global__ __launch_bounds__(1024) void norm_long_rows_bwd_kernel(NormBwdArgs a)
{
    __shared__ float part[32];
    RowSum<1024> total{part};
    const Row<DT, 1024> r(a.c);
    const int K = (a.c + 8191) / 8192;
    const uint64_t counter = a.drop.base();
    for (long row = blockIdx.x; row < a.n; row += gridDim.x) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        float sg = 0.f, sgh = 0.f, gamma[8];
        Words<DT, 8> vy, vs, vd;
        auto both = [&](int k) {
            r.load(r.from(a.dy, row), 0, k, vy);
            r.load(r.from(a.s, row), 0, k, vs);
            r.fit(k, false, vy);
            r.fit(k, false, vs);
#pragma unroll
            for (int j = 0; j < 8; ++j) gamma[j] = a.gamma && r.channel(k) + j < a.c ? a.gamma[r.channel(k) + j] : 1.f;
        };
        for (int k = 0; k < K; ++k) {
            both(k);
            float t0 = 0.f, t1 = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float g = product(vy[j], gamma[j]);
                t0 += g;
                t1 += g * ((vs[j] - mean) * rstd);
            }
            sg += t0;
            sgh += t1;
        }
        const float mg = total(sg) / (float)a.c, mgh = total(sgh) / (float)a.c;
        for (int k = 0; k < K; ++k) {
            both(k);
            if (a.dsum.p) {
                r.load(r.from(a.dsum, row), 0, k, vd);
                r.fit(k, false, vd);
            }
            if (r.channel(k) < a.c) put_gradients<true>(r, a, counter, row, k, vy, vs, vd, gamma, mean, rstd, mg, mgh);
        }
    }
}

// dgamma and dbeta of rows too long for registers: a thread eight channels, blockIdx.y a share of the rows
template <int DT> __global__ __launch_bounds__(1024) void norm_long_rows_wgrad_kernel(NormBwdArgs a)
{
    const Row<DT, 1024> r(a.c);
    const long cp = norm_copy_floats(a.c) / 2;
    for (int k = blockIdx.x; k < (a.c + 8191) / 8192; k += gridDim.x) {
        float dg[8] = {}, db[8] = {};
        for (long row = blockIdx.y; row < a.n; row += gridDim.y) {
            Words<DT, 8> vy, vs;
            r.load(r.from(a.dy, row), 0, k, vy);
            r.load(r.from(a.s, row), 0, k, vs);
            const float mean = a.mean[row], rstd = a.rstd[row];
            r.fit(k, false, vy);
            r.fit(k, false, vs);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dg[j] += vy[j] * ((vs[j] - mean) * rstd);
                db[j] += vy[j];
            }
        }
        float *dgamma = gridDim.y == 1 ? a.dgamma : a.scratch + blockIdx.y * 2L * cp;
        float *dbeta = gridDim.y == 1 ? a.dbeta : a.scratch + (blockIdx.y * 2L + 1) * cp;
        if (dgamma) put_values(dgamma, a.c, r.channel(k), dg);
        if (dbeta) put_values(dbeta, a.c, r.channel(k), db);
    }
}

constexpr int kLongRow = 32768, kLongRowBwd = 16384;    // longer rows do not fit the registers of a workgroup

template <int N> using num = std::integral_constant<int, N>;

// f(G, K, T) for rows of c channels, forwards; far: rows so far apart that 32 bits do not span those of a wave
template <class F> void pick_rows(int c, bool far, F f)
{
    if (c <= 8 && !far) return f(num<1>{}, num<1>{}, num<256>{});
    if (c <= 64 && !far) return f(num<8>{}, num<1>{}, num<256>{});
    if (c <= 128 && !far) return f(num<16>{}, num<1>{}, num<256>{});
    if (c <= 256 && !far) return f(num<32>{}, num<1>{}, num<256>{});
    if (c <= 512) return f(num<64>{}, num<1>{}, num<256>{});
    if (c <= 1024) return f(num<64>{}, num<2>{}, num<256>{});
    if (c <= 2048) return f(num<64>{}, num<4>{}, num<256>{});
    if (c <= 4096) return f(num<256>{}, num<2>{}, num<256>{});
    if (c <= 8192) return f(num<256>{}, num<4>{}, num<256>{});
    if (c <= 16384) return f(num<1024>{}, num<2>{}, num<1024>{});
    return f(num<1024>{}, num<4>{}, num<1024>{});
}

// the same backwards, where a lane also holds gamma and two sums a channel
template <class F> void pick_rows_bwd(int c, bool far, F f)
{
    if (c <= 8 && !far) return f(num<1>{}, num<1>{}, num<512>{});
    if (c <= 64 && !far) return f(num<8>{}, num<1>{}, num<512>{});
    if (c <= 128 && !far) return f(num<16>{}, num<1>{}, num<512>{});
    if (c <= 256 && !far) return f(num<32>{}, num<1>{}, num<512>{});
    if (c <= 512) return f(num<64>{}, num<1>{}, num<512>{});
    if (c <= 1024) return f(num<64>{}, num<2>{}, num<512>{});
    if (c <= 2048) return f(num<128>{}, num<2>{}, num<512>{});
    if (c <= 4096) return f(num<256>{}, num<2>{}, num<512>{});
    if (c <= 8192) return f(num<512>{}, num<2>{}, num<512>{});
    return f(num<1024>{}, num<2>{}, num<1024>{});
}

template <class F> void pick_type(int dtype, F f)
{
    if (dtype == 0) return f(num<0>{});
    if (dtype == 1) return f(num<1>{});
    return f(num<2>{});
}

// Sixteen columns a workgroup: four lanes take a float4 each and 64 groups of them share the copies out, eight loads in flight; latency is all there is
// to it (1024 copies of 128 floats in workgroups of 64 columns and 16 groups: 9.2 us).
__global__ __launch_bounds__(256) void norm_reduce_kernel(const float *scratch, int copies, float *dgamma, float *dbeta, int c)
{
    typedef float floatx4 __attribute__((ext_vector_type(4)));
    __shared__ floatx4 sh[4][4];
    const int cp = (c + 3) / 4 * 4, group = threadIdx.x >> 2;
    for (int first = blockIdx.x * 16; first < 2 * cp; first += gridDim.x * 16) {        // (every thread alike)
        const int e = first + 4 * (threadIdx.x & 3);
        floatx4 s{};
        if (e < 2 * cp) {
            const float *p = scratch + e;
            int i = group;
            for (; i + 7 * 64 < copies; i += 8 * 64) {
                floatx4 v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] = *reinterpret_cast<const floatx4 *>(p + (long)(i + 64 * u) * 2 * cp);
                s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
            }
            for (; i < copies; i += 64) s += *reinterpret_cast<const floatx4 *>(p + (long)i * 2 * cp);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = sum_over_groups<4>(s[j]);
        if ((threadIdx.x & 63) < 4) sh[threadIdx.x >> 6][threadIdx.x & 3] = s;
        __syncthreads();
        if (threadIdx.x < 4 && e < 2 * cp) {
            s = (sh[0][threadIdx.x] + sh[1][threadIdx.x]) + (sh[2][threadIdx.x] + sh[3][threadIdx.x]);
            float *out = e < cp ? dgamma : dbeta;
            const int k = e < cp ? e : e - cp;
            if (out)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (k + j < c) out[k + j] = s[j];
        }
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_norm_reduce(const float *scratch, int copies, float *dgamma, float *dbeta, int c, hipStream_t stream)
{
    norm_reduce_kernel<<<norm_blocks(norm_copy_floats(c), 16), 256, 0, stream>>>(scratch, copies, dgamma, dbeta, c);
    return hipGetLastError();
}

hipError_t launch_norm_rows(const NormArgs &a, hipStream_t stream)
{
    if (a.relu) return hipErrorInvalidValue;            // (a net's layers are maps)
    const bool adds = a.residual.p || a.sum.p || a.drop.thresh, far = far_apart({&a.x, &a.residual, &a.sum, &a.y});
    pick_type(a.dtype, [&](auto dt) {
        if (a.c > kLongRow) {
            norm_long_rows_kernel<dt()><<<norm_blocks(a.n, 1), 1024, 0, stream>>>(a);
            return;
        }
        pick_rows(a.c, far, [&](auto g, auto k, auto t) {
            if (adds) norm_rows_kernel<dt(), g(), k(), t(), true><<<norm_blocks(a.n, t() / g()), t(), 0, stream>>>(a);
            else norm_rows_kernel<dt(), g(), k(), t(), false><<<norm_blocks(a.n, t() / g()), t(), 0, stream>>>(a);
        });
    });
    return hipGetLastError();
}

// Where ROLES take the work: up to 512 rows, 1024 of more than 2048 channels.  With roles and with copies and a second launch, us, bf16: 1 x 777 3.4 and 5.0, 37 x
// 777 4.3 and 8.5, 512 x 777 7.2 and 9.0, 512 x 64 4.9 and 6.5, 1024 x 4096 11.2 and 21.3; 1024 x 777 10.9 and 9.6, 2048 x 64 11.3 and 6.7, 2048 x 4096 23.9
// and 22.5.
static bool takes_roles(const NormSpan &s) { return s.c > 8 && s.c <= kLongRowBwd && s.n <= (s.c > 2048 ? 1024 : 512); }

// (rows far apart take as many: their workgroups hold no more of them)
int norm_rows_bwd_copies(const NormSpan &s)
{
    if (s.c > kLongRowBwd) return (int)std::min<long>(s.n, 16);
    int copies = 1;
    if (takes_roles(s)) return copies;
    pick_rows_bwd(s.c, false, [&](auto g, auto, auto t) {
        const long rounds = (s.n + t() / g() - 1) / (t() / g());
        copies = (int)std::min<long>(rounds, 256 * 1024 / t());
    });
    return copies;
}

hipError_t launch_norm_rows_bwd(const NormBwdArgs &a, int copies, hipStream_t stream)
{
    if (a.relu_x) return hipErrorInvalidValue;
    const bool sums = a.dgamma || a.dbeta, results = a.dx.p || a.dresidual.p, adds = a.dsum.p || a.dresidual.p || a.drop.thresh;
    const bool far = far_apart({&a.dy, &a.s, &a.dsum, &a.dx, &a.dresidual});
    Launches done;
    pick_type(a.dtype, [&](auto dt) {
        if (a.c > kLongRowBwd) {
            if (sums) {
                norm_long_rows_wgrad_kernel<dt()><<<dim3((unsigned)std::min((a.c + 8191) / 8192, 65536), copies), 1024, 0, stream>>>(a);
                if (done.failed() || (copies > 1 && done.failed(launch_norm_reduce(a.scratch, copies, a.dgamma, a.dbeta, a.c, stream)))) return;
            }
            if (results) norm_long_rows_bwd_kernel<dt()><<<norm_blocks(a.n, 1), 1024, 0, stream>>>(a);
            return;
        }
        pick_rows_bwd(a.c, far, [&](auto g, auto k, auto t) {
            const long rounds = (a.n + t() / g() - 1) / (t() / g());
            const int all = (int)std::min<long>(rounds, 256 * 1024 / t());
            const bool roles = sums && takes_roles(a);
            if (roles) {
                const int walkers = results && !a.in_place() ? all : 0, blocks = walkers + (a.c + 63) / 64;
                if (adds) norm_rows_bwd_kernel<dt(), g(), k(), t(), true, true><<<blocks, t(), 0, stream>>>(a, walkers);
                else norm_rows_bwd_kernel<dt(), g(), k(), t(), false, true><<<blocks, t(), 0, stream>>>(a, walkers);
                if (done.failed() || walkers || !results) return;
            }
            NormBwdArgs b = a;
            if (roles) b.dgamma = b.dbeta = nullptr;
            if (roles || !sums) copies = all;
            if (adds) norm_rows_bwd_kernel<dt(), g(), k(), t(), true, false><<<copies, t(), 0, stream>>>(b, copies);
            else norm_rows_bwd_kernel<dt(), g(), k(), t(), false, false><<<copies, t(), 0, stream>>>(b, copies);
            if (!done.failed() && sums && !roles && copies > 1) done.failed(launch_norm_reduce(a.scratch, copies, a.dgamma, a.dbeta, a.c, stream));
        });
    });
    return done.status();
}

}  // namespace sk
