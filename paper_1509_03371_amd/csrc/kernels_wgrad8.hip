// Weight gradient of an inner product over inputs held in 8 bits: dw[o][k] = sum over positions q of dy[q][o] x[q][k].
#include "act8_device.h"
#include "reduce_copies.h"

namespace sk {

namespace {

typedef uint32_t words4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

// What a code stands for is exact in bf16, and so x goes to the matrix unit; dy goes there as bf16 terms that add up to it.  fp16 has 11 bits, two terms of
// 8; fp32 24, three.  Each term is cut off, not rounded, so what is left is exact and no term overflows; an infinite value has no rest.
template <int DT> constexpr int terms = DT == 1 ? 1 : DT == 2 ? 2 : 3;

// A workgroup's tile: TM x TN output and input channels, KS positions at a time, WM x WN waves.  BIG ones take half as many bytes from the caches for each product and
// keep two steps in LDS; small ones are for few weights or few positions.
struct Tile8 {
    int tm, tn;
    bool big;
};
template <int DT, bool BIG> constexpr int step_of = BIG && terms<DT> > 1 ? 32 : 64;      // positions; two steps of fp32's terms fit the LDS at 32
int step_positions(int dtype, bool big) { return big && dtype != 1 ? 32 : 64; }

struct Plan8 {
    Tile8 tile;
    long tiles_m, tiles_n, plane_steps, steps, splits;
};

Plan8 plan_of(const NormSpan &s, long c_out)
{
    Plan8 p;
    auto lay = [&](int tm, int tn, bool big, long fill) {
        const int ks = step_positions(s.dtype, big);
        p.tile = {tm, tn, big};
        p.plane_steps = (s.plane + ks - 1) / ks;
        p.steps = s.layout == ROWS ? (s.n + ks - 1) / ks : s.n * p.plane_steps;
        p.tiles_m = (c_out + tm - 1) / tm;
        p.tiles_n = (s.c + tn - 1) / tn;
        const long tiles = p.tiles_m * p.tiles_n, most = std::max<long>(1, p.steps / 4);       // four steps a workgroup or more
        p.splits = std::min(most, std::max<long>(1, fill / tiles));
        return tiles * p.splits;
    };
    // As many workgroups as fill the card: one a CU of big ones (bf16 takes small ones, see the kernel), else two.  Big ones where they fill half the card or more with
    // four copies of the gradient at most.  us with big and with small ones, fp16 (fp32): 2048 x 2048 weights over 8192 rows 184 and 219 (247 and 310), over 4096 120 and 134 (150 and
    // 181), over 1024 72 and 73 (80 and 83); with more copies 512 x 1024 over 128^2 pixels 59 and 60 (81 and 84), 512 x 512 over 65536 rows 91 and 102 (123 and 154), 256 x 256 over as
    // many 43 and 38 (52 and 50).  The rule leaves up to a quarter there; and over 300 rows, a few steps, small ones would take 20 of its 66 us.
    if (s.dtype != 1 && c_out >= 256 && s.c >= 256 && lay(256, 256, true, 256) >= 128 && p.splits <= 4) return p;
    const int tm = c_out <= 64 ? 64 : 128, tn = s.c <= 64 ? 64 : 128;
    // (three a CU where the tile is small: 200 x 48 weights over 512^2 pixels 42 us with two and 39 with three; 512 x 1024 over 128^2 62 and 78)
    const long fill = tm + tn < 256 ? 768 : 512;
    if (lay(tm, tn, false, fill) < 256) lay(64, 64, false, 512);
    return p;
}
long copy_floats(const NormSpan &s, long c_out) { return (c_out * (s.c + 1) + 3) / 4 * 4; }

struct Wgrad8Launch : Wgrad8Args {
    long tiles_n, tiles, steps, splits, plane_steps, copy;
    long dy_end, codes_end;                             // bytes that the operands span
    float *to;                                          // dw, or the copies of it
};

// 32 values of a line: codes or dy, as read
template <int B> struct Unit {                          // B bytes a value
    uint32_t w[8 * B];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < 8 * B; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void vectors(const char *p)
    {
        typedef uint32_t Four __attribute__((ext_vector_type(4), aligned(1)));
#pragma unroll
        for (int i = 0; i < 2 * B; ++i) {
            const Four v = reinterpret_cast<const Four *>(p)[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[4 * i + j] = v[j];
        }
    }
    // the values from `by` bytes on, zeros behind them
    __device__ __forceinline__ void down(int by)
    {
#pragma unroll
        for (int step = 4 * B; step >= 1; step /= 2)
#pragma unroll
            for (int i = 0; i < 8 * B; ++i) w[i] = (by / 4) & step ? (i + step < 8 * B ? w[i + step < 8 * B ? i + step : 0] : 0) : w[i];
        if (B < 4)
#pragma unroll
            for (int i = 0; i < 8 * B; ++i) w[i] = __builtin_amdgcn_alignbyte(i + 1 < 8 * B ? w[i + 1 < 8 * B ? i + 1 : 0] : 0, w[i], by & 3);
    }
    // `count` values at `off` of an operand that spans `end` bytes.  Whole vectors where the operand goes on for as long (what they bring behind `count` is
    // some other value of it), else its last ones, moved down.
    __device__ __forceinline__ void load(const char *base, long off, long end, int count)
    {
        if (off + 32 * B <= end) {
            vectors(base + off);
        } else if (end >= 32 * B) {
            vectors(base + end - 32 * B);
            down((int)(off + 32 * B - end));
        } else {                                        // an operand of fewer than 32 values
            clear();
#pragma unroll 1
            for (int j = 0; j < count; ++j) {
                const char *p = base + off + B * j;
                const uint32_t v = B == 1 ? *reinterpret_cast<const uint8_t *>(p) : B == 2 ? *reinterpret_cast<const uint16_t *>(p) : *reinterpret_cast<const uint32_t *>(p);
#pragma unroll
                for (int i = 0; i < 8 * B; ++i) w[i] |= i == B * j / 4 ? v << 8 * (B * j % 4) : 0;
            }
        }
    }
    // zeros behind `count`: positions that are not there must not reach the sums
    __device__ __forceinline__ void keep(int count)
    {
#pragma unroll
        for (int i = 0; i < 8 * B; ++i) {
            const int left = (count * B - 4 * i) * 8;
            w[i] = left >= 32 ? w[i] : left <= 0 ? 0 : w[i] & ((1u << left) - 1);
        }
    }
};

template <int CODE> __device__ __forceinline__ void widen(const Unit<1> &u, float scale, words4 (&to)[4])
{
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (CODE == E4M3) {
            to[i / 2][2 * (i % 2)] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u.w[i], scale, false));
            to[i / 2][2 * (i % 2) + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u.w[i], scale, true));
        } else {
            float f[4];
            Code8<CODE>::numbers(u.w[i], scale, f);
            odd |= Code8<CODE>::unlike(u.w[i]);
            // exact: the upper halves are the values
            to[i / 2][2 * (i % 2)] = __builtin_amdgcn_perm(__float_as_uint(f[1]), __float_as_uint(f[0]), 0x07060302);
            to[i / 2][2 * (i % 2) + 1] = __builtin_amdgcn_perm(__float_as_uint(f[3]), __float_as_uint(f[2]), 0x07060302);
        }
    }
    if (odd)
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if ((u.w[i / 4] >> 8 * (i % 4) & 0xff) == Code8<CODE>::nan) to[i / 8][i / 2 % 4] |= 0x7fc0u << 16 * (i % 2);
}

__device__ __forceinline__ float rest(float v) { return magnitude(v) == 0x7f800000u ? 0.f : v - __uint_as_float(__float_as_uint(v) & 0xffff0000u); }

// term n of the unit's values
template <int DT> __device__ __forceinline__ void term(Unit<DT == 0 ? 4 : 2> &u, int n, words4 (&to)[4])
{
    if constexpr (DT == 1) {
#pragma unroll
        for (int i = 0; i < 16; ++i) to[i / 4][i % 4] = u.w[i];
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float a, b;
            if constexpr (DT == 2) {
                a = (float)__builtin_bit_cast(_Float16, (uint16_t)u.w[i]);
                b = (float)__builtin_bit_cast(_Float16, (uint16_t)(u.w[i] >> 16));
                if (n == 1) {
                    a = rest(a);
                    b = rest(b);
                }
            } else {
                a = __uint_as_float(u.w[2 * i]);
                b = __uint_as_float(u.w[2 * i + 1]);
                u.w[2 * i] = __float_as_uint(rest(a));              // for the next term
                u.w[2 * i + 1] = __float_as_uint(rest(b));
            }
            to[i / 4][i % 4] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302);
        }
    }
}

// Lane l of a fragment holds channel l % 16 at eight of 32 positions; which eight is the same for both operands, and that is all that matters.  MAPS keep a channel's
// positions side by side in LDS.  ROWS keep a position's channels side by side, and a transposing read makes of four positions' sixteen channels
// (lane 4 r + p of sixteen names position r, channels 4 p ..) each channel's four positions: those at 4 g .. and at 16 + 4 g .. for group g of sixteen lanes, which
// lie in as many banks as there are.
template <bool IS_ROWS> __device__ __forceinline__ bf16x8 fragment(const char *lds, int pitch, int channel, int position)
{
    const int lane = threadIdx.x & 63, g = lane >> 4, l = lane & 15;
    if constexpr (IS_ROWS) {
        typedef shortx4 __attribute__((address_space(3))) *lds_s4;
        const char *at = lds + (position + 4 * g + (l >> 2)) * pitch + 2 * channel + 8 * (l & 3);
        const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)at);
        const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(at + 16 * pitch));
        typedef short shortx8 __attribute__((ext_vector_type(8)));
        return __builtin_bit_cast(bf16x8, shortx8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    } else {
        return *reinterpret_cast<const bf16x8 *>(lds + (channel + l) * pitch + 2 * position + 16 * g);
    }
}

// A workgroup takes TM x TN weights and a share of the positions, KS at a time: its threads load 32 values of a line each (of x a block with its scale), a step
// ahead, widen them on their way into LDS, and its waves multiply, a part of the tile each.  db comes out of the same fragments, times ones.
// 16384 rows, 2048 x 4096 weights, 275 GFLOP: bf16 and e4m3 349 us = 0.79 PFLOP/s, int8 395 (a library product of bf16 tensors 231: 1.19), passes one after another; the
// first hundred or so after a pause take up to 430.  Waves that multiply go first (s_setprio): 398 without.  Of a CU's clocks the matrix units work in 31 of 100 and the LDS in 46 (for 32
// positions of a tile it moves 48 KB, one and a half times as long as the products take, a third of it banks in conflict); the rest waits, for the loads of a step, of
// which one is under way, for one another and for the LDS.  Three workgroups a CU at 160 registers cover for one another, two (240 registers) take 483 us, steps of 32 positions
// 464, 256 x 128 tiles of four waves with two steps under way 668.  fp16 and fp32 have two and three products for each load, and there BIG tiles pay: fp16 608 us and 655
// with small ones (bf16 422 and 349).
template <int DT, int CODE, bool IS_ROWS, int TM, int TN, bool BIG> __global__ __launch_bounds__(BIG ? 512 : 256, 2) void wgrad8_kernel(Wgrad8Launch a)
{
    constexpr int NS = terms<DT>, B = DT == 0 ? 4 : 2, T = BIG ? 512 : 256, KS = step_of<DT, BIG>;
    constexpr int WN = 2, WM = T / 64 / WN, IM = TM / WM / 16, IN = TN / WN / 16;       // waves; 16 x 16 fragments of a wave
    constexpr int per = KS / 32;                        // blocks of a map's line in a step
    constexpr int pitch_m = IS_ROWS ? 2 * TM + 32 : 2 * KS + 16, pitch_n = IS_ROWS ? 2 * TN + 32 : 2 * KS + 16;
    constexpr int plane_m = (IS_ROWS ? KS : TM) * pitch_m, plane_n = (IS_ROWS ? KS : TN) * pitch_n, buffer = NS * plane_m + plane_n;
    extern __shared__ words4 smem8[];
    char *const smem = reinterpret_cast<char *>(smem8);
    const unsigned block = neighbour();
    const long split = block / a.tiles, tile = block - split * a.tiles;
    const long m0 = tile / a.tiles_n * TM, n0 = tile % a.tiles_n * TN;
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wm = wave / WN * (TM / WM), wn = wave % WN * (TN / WN);
    const bool bias = a.db && n0 == 0 && wn == 0;

    // this thread's units: of dy, and of x from the other end of the workgroup
    const int um = threadIdx.x, un = T - 1 - threadIdx.x;
    const bool has_m = um < TM * per, has_n = un < TN * per;
    Unit<B> dy;
    Unit<1> x;
    uint32_t scale = 0;
    // Where they lie: a part of the thread's own that stays, and one of the step's that all share and the scalar unit keeps.
    const long om = IS_ROWS ? m0 + 32 * (um % (TM / 32)) : std::min(m0 + um / per, a.c_out - 1);
    const long kn = IS_ROWS ? n0 + 32 * (un % (TN / 32)) : std::min<long>(n0 + un / per, a.c - 1);
    const int row_m = um / (TM / 32), row_n = un / (TN / 32), px_m = 32 * (um % per), px_n = 32 * (un % per);
    const long at_dy = B * (IS_ROWS ? row_m * a.dy.sn + om : om * a.dy.sc + px_m);
    const long at_x = IS_ROWS ? row_n * a.x.sn + kn : kn * a.x.sc + px_n, at_scale = IS_ROWS ? row_n * a.x.ssn + kn / 32 : kn * a.x.ssc + px_n / 32;
    const long first = a.steps * split / a.splits, last = a.steps * (split + 1) / a.splits;
    long b = IS_ROWS ? 0 : first / a.plane_steps, q0 = IS_ROWS ? first * KS : (first - b * a.plane_steps) * KS;      // image; row or pixel
    auto fetch = [&] {                                  // the next step's
        const long left = (IS_ROWS ? a.n : a.plane) - q0;
        const long dy0 = IS_ROWS ? q0 * a.dy.sn : b * a.dy.sn + q0, x0 = IS_ROWS ? q0 * a.x.sn : b * a.x.sn + q0;
        const long scale0 = IS_ROWS ? q0 * a.x.ssn : b * a.x.ssn + q0 / 32;
        const int some = left < KS ? (int)left : KS;    // rows, or pixels, of the step
        if (has_m) {
            const int count = IS_ROWS ? (row_m < some && om < a.c_out ? (int)std::min<long>(32, a.c_out - om) : 0) : std::min(32, some - px_m);
            if (count > 0) {
                dy.load(static_cast<const char *>(a.dy.p), B * dy0 + at_dy, a.dy_end, count);
                if (!IS_ROWS && count < 32) dy.keep(count);
            } else {
                dy.clear();
            }
        }
        if (has_n) {
            const int count = IS_ROWS ? (row_n < some && kn < a.c ? (int)std::min<long>(32, a.c - kn) : 0) : std::min(32, some - px_n);
            if (count > 0) {
                x.load(reinterpret_cast<const char *>(a.x.codes), x0 + at_x, a.codes_end, count);
                if (!IS_ROWS && count < 32) x.keep(count);
                scale = a.x.scales[scale0 + at_scale];
            } else {
                x.clear();
                scale = 127;
            }
        }
        q0 += KS;
        if (!IS_ROWS && q0 >= a.plane) {
            q0 = 0;
            ++b;
        }
    };
    auto put = [&](char *lds) {
        words4 w[4];
        if (has_m) {
            char *at = lds + (IS_ROWS ? um / (TM / 32) * pitch_m + 64 * (um % (TM / 32)) : um / per * pitch_m + 64 * (um % per));
#pragma unroll
            for (int n = 0; n < NS; ++n) {
                term<DT>(dy, n, w);
#pragma unroll
                for (int i = 0; i < 4; ++i) *reinterpret_cast<words4 *>(at + n * plane_m + 16 * i) = w[i];
            }
        }
        if (has_n) {
            char *at = lds + NS * plane_m + (IS_ROWS ? un / (TN / 32) * pitch_n + 64 * (un % (TN / 32)) : un / per * pitch_n + 64 * (un % per));
            widen<CODE>(x, Code8<CODE>::scale(scale), w);
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<words4 *>(at + 16 * i) = w[i];
        }
    };

    floatx4 acc[IM][IN], ones_acc[IM];
#pragma unroll
    for (int i = 0; i < IM; ++i) {
        ones_acc[i] = floatx4{};
#pragma unroll
        for (int j = 0; j < IN; ++j) acc[i][j] = floatx4{};
    }
    bf16x8 ones;
#pragma unroll
    for (int j = 0; j < 8; ++j) ones[j] = (__bf16)1.f;
    auto multiply = [&](const char *lds) {
#pragma unroll
        for (int h = 0; h < KS; h += 32) {
            bf16x8 v[IN];
#pragma unroll
            for (int j = 0; j < IN; ++j) v[j] = fragment<IS_ROWS>(lds + NS * plane_m, pitch_n, wn + 16 * j, h);
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int i = 0; i < IM; ++i) {
                    const bf16x8 u = fragment<IS_ROWS>(lds + n * plane_m, pitch_m, wm + 16 * i, h);
#pragma unroll
                    for (int j = 0; j < IN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u, v[j], acc[i][j], 0, 0, 0);
                    if (bias) ones_acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u, ones, ones_acc[i], 0, 0, 0);
                }
        }
    };
    fetch();
    if constexpr (BIG) {
        put(smem);
        if (first + 1 < last) fetch();
        int now = 0;
        for (long step = first; step < last; ++step) {
            __syncthreads();                            // this step is in LDS, and the one before has been read
            if (step + 1 < last) put(smem + (now ^ 1) * buffer);
            if (step + 2 < last) fetch();
            __builtin_amdgcn_s_setprio(1);
            multiply(smem + now * buffer);
            __builtin_amdgcn_s_setprio(0);
            now ^= 1;
        }
    } else {
        for (long step = first; step < last; ++step) {
            __syncthreads();                            // the step before has been read
            put(smem);
            __syncthreads();
            if (step + 1 < last) fetch();
            __builtin_amdgcn_s_setprio(1);
            multiply(smem);
            __builtin_amdgcn_s_setprio(0);
        }
    }
    // lane l of a result holds column l % 16 of rows 4 (l / 16) ..
    float *const dw = a.to + split * a.copy, *const db = a.splits > 1 ? dw + a.c_out * a.c : a.db;
    const bool add = a.splits == 1 && a.accumulate;
#pragma unroll
    for (int i = 0; i < IM; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const long o = m0 + wm + 16 * i + 4 * (lane >> 4) + r;
            if (o >= a.c_out) continue;
#pragma unroll
            for (int j = 0; j < IN; ++j) {
                const long k = n0 + wn + 16 * j + (lane & 15);
                if (k < a.c) {
                    float *at = dw + o * a.c + k;
                    *at = add ? *at + acc[i][j][r] : acc[i][j][r];
                }
            }
            if (bias && (lane & 15) == 0) db[o] = add ? db[o] + ones_acc[i][r] : ones_acc[i][r];
        }
}

// dw and db (side by side in each copy) from the copies, or from none
__global__ __launch_bounds__(256) void wgrad8_reduce_kernel(Wgrad8Launch a)
{
    __shared__ float sh[16][64];
    const long weights = a.c_out * a.c, all = weights + (a.db ? a.c_out : 0);
    for (long first = blockIdx.x * 64L; first < all; first += gridDim.x * 64L) {       // (every thread alike)
        const long left = a.copy - first;
        const float v = sum_copies64(a.scratch + first, a.copy, 0, (int)std::min<long>(left, 64), (int)a.splits, sh);
        const long e = first + threadIdx.x;
        if (threadIdx.x < 64 && e < all) {
            float *at = e < weights ? a.dw + e : a.db + (e - weights);
            *at = a.accumulate ? *at + v : v;
        }
        __syncthreads();
    }
}

__global__ __launch_bounds__(256) void wgrad8_clear_kernel(float *dw, float *db, long weights, long c_out)
{
    const long all = weights + (db ? c_out : 0);
    for (long e = blockIdx.x * 256L + threadIdx.x; e < all; e += gridDim.x * 256L) (e < weights ? dw[e] : db[e - weights]) = 0.f;
}

template <int N> using num = std::integral_constant<int, N>;

template <class F> void pick_tile(const Tile8 &t, F f)
{
    typedef std::true_type Big;
    typedef std::false_type Small;
    if (t.big) return f(num<256>{}, num<256>{}, Big{});
    if (t.tm == 128 && t.tn == 128) return f(num<128>{}, num<128>{}, Small{});
    if (t.tm == 128) return f(num<128>{}, num<64>{}, Small{});
    if (t.tn == 128) return f(num<64>{}, num<128>{}, Small{});
    return f(num<64>{}, num<64>{}, Small{});
}

// bytes of LDS, as the kernel lays it out
template <int DT, bool IS_ROWS, int TM, int TN, bool BIG> constexpr int lds_bytes()
{
    constexpr int KS = step_of<DT, BIG>;
    return (BIG ? 2 : 1) * (IS_ROWS ? KS * (terms<DT> * (2 * TM + 32) + 2 * TN + 32) : (2 * KS + 16) * (terms<DT> * TM + TN));
}

}  // namespace

size_t wgrad8_scratch_floats(const NormSpan &s, long c_out)
{
    if (s.n * s.plane == 0) return 0;
    const Plan8 p = plan_of(s, c_out);
    return p.splits > 1 ? (size_t)(p.splits * copy_floats(s, c_out)) : 0;
}

hipError_t launch_wgrad8(const Wgrad8Args &given, hipStream_t stream)
{
    Wgrad8Launch a;
    static_cast<Wgrad8Args &>(a) = given;
    const long weights = a.c_out * a.c;
    if (a.n * a.plane == 0) {
        if (!a.accumulate) wgrad8_clear_kernel<<<norm_blocks(weights + a.c_out, 256), 256, 0, stream>>>(a.dw, a.db, weights, a.c_out);
        return hipGetLastError();
    }
    const Plan8 p = plan_of(a, a.c_out);
    a.tiles_n = p.tiles_n; a.tiles = p.tiles_m * p.tiles_n; a.steps = p.steps; a.splits = p.splits;
    a.plane_steps = p.plane_steps;
    a.copy = copy_floats(a, a.c_out);
    a.to = p.splits > 1 ? a.scratch : a.dw;
    const bool rows = a.layout == ROWS;
    const long size = a.dtype == 0 ? 4 : 2;
    a.dy_end = size * ((a.n - 1) * a.dy.sn + (rows ? a.c_out : (a.c_out - 1) * a.dy.sc + a.plane));
    a.codes_end = (a.n - 1) * a.x.sn + (rows ? a.c : (a.c - 1L) * a.x.sc + a.plane);
    if (a.tiles * a.splits > 0x7fffffffL) return hipErrorInvalidValue;
    const unsigned blocks = (unsigned)(a.tiles * a.splits);
    Launches done;
    auto type = [&](auto dt) {
        pick_code(a.x.code, [&](auto code) {
            pick_tile(p.tile, [&](auto tm, auto tn, auto big) {
                auto go = [&](auto is_rows) {
                    constexpr int lds = lds_bytes<dt(), is_rows(), tm(), tn(), big()>();
                    auto *kernel = wgrad8_kernel<dt(), code(), is_rows(), tm(), tn(), big()>;
                    if (lds > 65536 && done.failed(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds))) return;
                    kernel<<<blocks, big() ? 512 : 256, lds, stream>>>(a);
                };
                if (rows) go(std::true_type{});
                else go(std::false_type{});
            });
        });
    };
    if (a.dtype == 0) type(num<0>{});
    else if (a.dtype == 1) type(num<1>{});
    else type(num<2>{});
    if (done.failed() || p.splits == 1) return done.status();
    wgrad8_reduce_kernel<<<norm_blocks(weights + a.c_out, 64), 256, 0, stream>>>(a);
    return done.status();
}

}  // namespace sk
