// add_norm.hip -- root-mean-square norm of rows with the residual's addition,
// an 8-bit output and dropout, its gradients, and dropout alone (finc_add_norm_*,
// finc_dropout of finc.h).
//
// Every value is read once and written once: bound by memory.  A row lives in
// the registers of 16 lanes, a wave, or a workgroup, by its width; r, its mean
// square, the output and its largest value come from one pass.  Rows of one
// group follow each other in a loop that keeps w (and, for the gradients, dw) in
// registers.
#include <type_traits>

#include "seq_common.h"

namespace {

using namespace finc_seq;

// ---- the generator ---------------------------------------------------------------

struct Drop {
    unsigned long long seed, offset;
    unsigned cut;   // 0: no dropout
    float scale;
};

// Eight elements of sixteen random bits: Philox4x32-10 at counter `at`.
__device__ inline void drop_bits(const Drop &d, unsigned long long at, unsigned (&w)[4]) {
    at += d.offset;
    unsigned c0 = (unsigned)at, c1 = (unsigned)(at >> 32), c2 = 0, c3 = 0;
    unsigned k0 = (unsigned)d.seed, k1 = (unsigned)(d.seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const unsigned long long p = (unsigned long long)c0 * 0xD2511F53u;
        const unsigned long long q = (unsigned long long)c2 * 0xCD9E8D57u;
        c0 = (unsigned)(q >> 32) ^ c1 ^ k0;
        c1 = (unsigned)q;
        c2 = (unsigned)(p >> 32) ^ c3 ^ k1;
        c3 = (unsigned)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    w[0] = c0;
    w[1] = c1;
    w[2] = c2;
    w[3] = c3;
}
// Which of eight elements are kept.
__device__ inline unsigned kept_bits(const Drop &d, unsigned long long at) {
    unsigned w[4], kept = 0;
    drop_bits(d, at, w);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        kept |= (unsigned)((i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu) >= d.cut) << i;
    return kept;
}
__device__ inline void drop(const Drop &d, unsigned long long at, float (&v)[8]) {
    unsigned w[4];
    drop_bits(d, at, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned u = i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu;
        v[i] = u < d.cut ? 0.0f : v[i] * d.scale;
    }
}

// ---- reductions over a row's lanes, the result in all of them ----------------------

template <int CTRL>
__device__ inline unsigned turn(unsigned v) {
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
struct Sum {
    static __device__ unsigned of(unsigned a, unsigned b) {
        return __builtin_bit_cast(unsigned,
                                  __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
    }
};
template <typename Op>
__device__ inline unsigned all16(unsigned v) {
    v = Op::of(v, turn<0x128>(v));   // row_ror:8, 4, 2, 1
    v = Op::of(v, turn<0x124>(v));
    v = Op::of(v, turn<0x122>(v));
    return Op::of(v, turn<0x121>(v));
}
template <typename Op>
__device__ inline unsigned all64(unsigned v) {
    v = all16<Op>(v);
    const unsigned a = (unsigned)__builtin_amdgcn_readlane((int)v, 0);
    const unsigned b = (unsigned)__builtin_amdgcn_readlane((int)v, 16);
    const unsigned c = (unsigned)__builtin_amdgcn_readlane((int)v, 32);
    const unsigned e = (unsigned)__builtin_amdgcn_readlane((int)v, 48);
    return Op::of(Op::of(a, b), Op::of(c, e));
}
// R lanes a row; above a wave through LDS (two buffers in turn, so that one barrier
// a reduction is enough).
template <typename Op, int R>
__device__ inline unsigned all_lanes(unsigned v, unsigned *lds, int &turn_of) {
    if (R == 16)
        return all16<Op>(v);
    v = all64<Op>(v);
    if (R == 64)
        return v;
    unsigned *buf = lds + (turn_of & 1) * (R / 64);
    ++turn_of;
    if ((threadIdx.x & 63) == 0)
        buf[threadIdx.x >> 6] = v;
    __syncthreads();
    // a wave's result in every row of lanes, 0 past the last wave
    const int i = threadIdx.x & 15;
    return all16<Op>(i < R / 64 ? buf[i] : 0u);
}
template <int R>
__device__ inline float sum_lanes(float v, unsigned *lds, int &turn_of) {
    return __builtin_bit_cast(float,
                              all_lanes<Sum, R>(__builtin_bit_cast(unsigned, v), lds, turn_of));
}

// Sums and largest magnitudes in 64 bits, the result in all lanes.
template <int CTRL>
__device__ inline double turn64(double v) {
    const unsigned long long b = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = turn<CTRL>((unsigned)b), hi = turn<CTRL>((unsigned)(b >> 32));
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
__device__ inline double lane64(double v, int lane) {
    const unsigned long long b = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)b, lane);
    const unsigned hi = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)(b >> 32), lane);
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
struct Sum64 {
    static __device__ double of(double a, double b) { return a + b; }
};
// By the bits without the sign: NaN is above infinity and stays.
struct Max64 {
    static __device__ double of(double a, double b) {
        const unsigned long long u = __builtin_bit_cast(unsigned long long, a) << 1;
        const unsigned long long v = __builtin_bit_cast(unsigned long long, b) << 1;
        return u > v ? a : b;
    }
};
template <typename Op>
__device__ inline double all16_64(double v) {
    v = Op::of(v, turn64<0x128>(v));
    v = Op::of(v, turn64<0x124>(v));
    v = Op::of(v, turn64<0x122>(v));
    return Op::of(v, turn64<0x121>(v));
}
template <typename Op, int R>
__device__ inline double all_lanes64(double v, double *lds, int &turn_of) {
    v = all16_64<Op>(v);
    if (R == 16)
        return v;
    v = Op::of(Op::of(lane64(v, 0), lane64(v, 16)), Op::of(lane64(v, 32), lane64(v, 48)));
    if (R == 64)
        return v;
    double *buf = lds + (turn_of & 1) * (R / 64);
    ++turn_of;
    if ((threadIdx.x & 63) == 0)
        buf[threadIdx.x >> 6] = v;
    __syncthreads();
    const int i = threadIdx.x & 15;
    return all16_64<Op>(i < R / 64 ? buf[i] : 0.0);
}

// 1 / sqrt(v) and 1 / v, from the hardware's first 24 bits by two steps of Newton's,
// without the scaling that the correctly rounded ones do near the range's ends.  At 0
// and infinity, where a step is NaN, the first value is the result.
__device__ inline double rsqrt64(double v) {
    const double first = __builtin_amdgcn_rsq(v);
    double y = first;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        y = __builtin_fma(0.5 * y, __builtin_fma(-v * y, y, 1.0), y);
    return y == y ? y : first;
}
__device__ inline double rcp64(double v) {
    const double first = __builtin_amdgcn_rcp(v);
    double y = first;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        y = __builtin_fma(y, __builtin_fma(-v, y, 1.0), y);
    return y == y ? y : first;
}

// y of the 8-bit norm, from r and what its rounding dropped.
__device__ inline double row_value(float r, float low, double inv, float w) {
    return ((double)r + (double)low) * inv * (double)w;
}

struct NormArgs {
    const void *x, *res, *dr;   // backward: x is dy, res is r
    void *y, *r;                // backward: y is dx, r is dresidual
    long long sx, sres, sy, sr, sdr;
    const float *w;
    float *scale, *partial;
    int M, D, per;              // per: vectors of 8 in a row
    double eps;
    Drop drop;
};

// Eight elements of a row from c on as they lie in memory, or its last eight where they
// would pass its end: all of a row's loads are under way before settle8() waits for the
// first, and the row's end is one load, not eight.  16384 x 2063 in bf16: 56 us forward and
// 103 the gradients, 73 and 126 with elements one by one and each vector waited for.
// TINY: rows of fewer than eight.
constexpr int kTinyThreads = 128;   // of a workgroup for them, and for no other rows
template <typename E>
using Raw8 = typename Vec<E, 8>::type;
template <bool TINY, typename E>
__device__ inline Raw8<E> load8(const E *row, int c, int D) {
    Raw8<E> t = {};
    if (!TINY) {
        if (c < D)   // lanes past the end would only load again what others do
            t = *(const Raw8<E> *)(row + min(c, D - 8));
        return t;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        t[i] = row[min(i, D - 1)];
    return t;
}
// Those of load8 at their places, 0 past the row's end.
template <bool TINY, typename E>
__device__ inline void settle8(Raw8<E> t, int c, int D, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = (float)t[i];
    if (TINY) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = keep_if(c + i < D, v[i]);
    } else if (c + 8 > D) {
        const int by = afresh(min(c + 8 - D, 8));
#pragma unroll
        for (int h = 8; h; h >>= 1)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = by & h ? (i + h < 8 ? v[i + h < 8 ? i + h : 0] : 0.0f) : v[i];
    }
}

// (mean r^2 + eps)^(-1/2) of a row whose squares leave fp32's range.
template <int R, int V>
__device__ inline float inv_wide(const float (&r)[V][8], int D, double eps, double *lds,
                                 int &turn_of) {
    double ss = 0.0;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            ss = __builtin_fma((double)r[v][i], (double)r[v][i], ss);
    ss = all_lanes64<Sum64, R>(ss, lds, turn_of);
    return (float)rsqrt64(__builtin_fma(ss, 1.0 / (double)afresh(D), eps));
}

// R lanes a row, V vectors of 8 a lane: vector v of a lane is lane + v R.  The mean square
// is in fp32, and again in fp64 for a row where it overflows or, below 2^-80, may have lost
// squares to underflow.  Asked of a scalar that costs nothing (32768 x 333 in bf16 18.7 us;
// by a comparison of lanes 19.7, in fp64 throughout 20.4).  Bound by memory: 32768 x 2048 in
// bf16 with an fp32 residual and dropout 150 us, 805 MB at 5.4 TB/s (the last-level cache
// holds some of them; a copy of 2 GiB reaches 4.8).
template <typename E, typename F, int R, int V, int TH>
__global__ __launch_bounds__(TH) void norm_forward_kernel(NormArgs a) {
    __shared__ unsigned lds[2 * (TH / 64)];
    __shared__ double lds64[2 * (TH / 64)];
    constexpr bool kTiny = TH == kTinyThreads;
    const int lane = threadIdx.x % R;
    int turn_of = 0, turn_of64 = 0;
    float w[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = (lane + v * R) * 8;
        settle8<kTiny, float>(load8<kTiny>(a.w, c, a.D), c, a.D, w[v]);
    }
    const float mean = 1.0f / (float)a.D, eps = (float)a.eps;
    const long long step = (long long)gridDim.x * (TH / R);
    // rows of a wave's other groups may be missing: they run on row M - 1 and do
    // not write
    for (long long m0 = (long long)blockIdx.x * (TH / R); m0 < a.M; m0 += step) {
        const long long mm = m0 + threadIdx.x / R;
        const bool live = mm < a.M;
        const long long m = live ? mm : a.M - 1;
        float r[V][8], ss = 0.0f;
        const E *x = (const E *)a.x + m * a.sx;
        const F *res = a.res ? (const F *)a.res + m * a.sres : nullptr;
        Raw8<E> tx[V];
        Raw8<F> tr[V] = {};
#pragma unroll
        for (int v = 0; v < V; ++v)
            tx[v] = load8<kTiny>(x, (lane + v * R) * 8, a.D);
        if (res)
#pragma unroll
            for (int v = 0; v < V; ++v)
                tr[v] = load8<kTiny>(res, (lane + v * R) * 8, a.D);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (lane + v * R) * 8;
            settle8<kTiny, E>(tx[v], c, a.D, r[v]);
            if (a.drop.cut && c < a.D)
                drop(a.drop, (unsigned long long)m * a.per + (lane + v * R), r[v]);
            if (res) {
                float t[8];
                settle8<kTiny, F>(tr[v], c, a.D, t);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    r[v][i] += t[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                ss = __builtin_fmaf(r[v][i], r[v][i], ss);
        }
        if (a.r && live) {
            F *out = (F *)a.r + m * a.sr;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = (lane + v * R) * 8;
                store_upto<F, 8>(out + c, a.D - c, r[v]);
            }
        }
        ss = sum_lanes<R>(ss, lds, turn_of);
        const float var = __builtin_fmaf(ss, mean, eps);
        float inv = rsqrtf(var);
        // 2^-80 <= var < inf by its bits, the same in all of the row's lanes
        int bits = __builtin_bit_cast(int, var);
        if (R >= 64)
            bits = __builtin_amdgcn_readfirstlane(bits);
        if (__builtin_expect((unsigned)bits - (47u << 23) >= (208u << 23), 0))
            inv = inv_wide<R, V>(r, a.D, a.eps, lds64, turn_of64);
        if (live) {
            E *out = (E *)a.y + m * a.sy;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = (lane + v * R) * 8;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    r[v][i] = r[v][i] * inv * w[v][i];
                store_upto<E, 8>(out + c, a.D - c, r[v]);
            }
        }
    }
}

// The same with the output in 8 bits.  An element takes another step of e4m3 than the
// definition's where its error crosses the middle of two: in fp32 a few in ten
// million.  So the sum (kept as an fp32 value and what that rounds off), the mean, the
// scale and the quotient are in fp64, and r keeps its low part: 32768 x 2048 in bf16 with
// the sum stored takes 137 us (bytes: 98), 93 in fp32; 64 x 1000 takes 5.6 (4.8).
template <typename E, typename F, int R, int V, int TH>
__global__ __launch_bounds__(TH) void norm_fp8_kernel(NormArgs a) {
    __shared__ double lds[2 * (TH / 64)];
    constexpr bool kKeep = V == 1;   // w in registers; the widest rows read it again
    const int lane = threadIdx.x % R;
    int turn_of = 0;
    const double mean = 1.0 / (double)a.D;
    const double factor = 65536.0 / (65536.0 - (double)a.drop.cut);
    float w[8];
    if (kKeep)
        load_upto<float, 8>(a.w + lane * 8, a.D - lane * 8, w);
    const long long step = (long long)gridDim.x * (TH / R);
    for (long long m0 = (long long)blockIdx.x * (TH / R); m0 < a.M; m0 += step) {
        const long long mm = m0 + threadIdx.x / R;
        const bool live = mm < a.M;
        const long long m = live ? mm : a.M - 1;
        float r[V][8], low[V][8];
        double ss = 0.0;
        const E *x = (const E *)a.x + m * a.sx;
        const F *res = a.res ? (const F *)a.res + m * a.sres : nullptr;
        const float *wr = a.w;
        asm volatile("" : "+s"(wr));   // read in every row, not once into registers
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (lane + v * R) * 8;
            float t[8];
            load_upto<E, 8>(x + c, a.D - c, r[v]);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                t[i] = 0.0f;
            if (res)
                load_upto<F, 8>(res + c, a.D - c, t);
            unsigned kept = 0xffu;
            if (a.drop.cut && c < a.D)
                kept = kept_bits(a.drop, (unsigned long long)m * a.per + (lane + v * R));
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double d = __builtin_fma((double)(kept >> i & 1 ? r[v][i] : 0.0f), factor,
                                               (double)t[i]);
                r[v][i] = (float)d;
                low[v][i] = (float)(d - (double)r[v][i]);
                ss = __builtin_fma(d, d, ss);
            }
        }
        if (a.r && live) {
            F *out = (F *)a.r + m * a.sr;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = (lane + v * R) * 8;
                store_upto<F, 8>(out + c, a.D - c, r[v]);
            }
        }
        ss = all_lanes64<Sum64, R>(ss, lds, turn_of);
        const double inv = rsqrt64(__builtin_fma(ss, mean, a.eps));
        double top = 0.0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (lane + v * R) * 8;
            if (!kKeep)
                load_upto<float, 8>(wr + c, a.D - c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                top = Max64::of(top, row_value(r[v][i], low[v][i], inv, w[i]));
        }
        top = all_lanes64<Max64, R>(top, lds, turn_of);
        double s = __builtin_fabs(top) * (1.0 / 448.0);
        s = s < 0x1p-126 ? 0x1p-126 : s;
        const double to = rcp64(s);
        if (!live)
            continue;
        if (lane == 0)
            a.scale[m] = (float)s;
        unsigned char *out = (unsigned char *)a.y + m * a.sy;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (lane + v * R) * 8;
            float y[8];
            if (!kKeep)
                load_upto<float, 8>(wr + c, a.D - c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                y[i] = (float)(row_value(r[v][i], low[v][i], inv, w[i]) * to);
            int q[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                q[h] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h], y[4 * h + 1], 0, false);
                q[h] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h + 2], y[4 * h + 3], q[h], true);
            }
            if (c + 8 <= a.D) {
                typedef int int2u __attribute__((ext_vector_type(2), aligned(1)));
                *(int2u *)(out + c) = int2u{q[0], q[1]};
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c + i < a.D)
                        out[c + i] = (unsigned char)(q[i >> 2] >> (8 * (i & 3)));
            }
        }
    }
}

// dr = dr_in + inv (w dy - r inv^2 mean(w dy r)), and the workgroup's sum of dw.
// Where w dy points along r the difference cancels, down to eps inv^2 of its terms:
// the two means and the difference are in fp64, whose multiply-adds issue at fp32's
// rate here and hide behind the memory: 25600 x 512 in fp32 in 32 us and 4 for dw's sum.
template <typename E, typename F, int R, int V, int TH>
__global__ __launch_bounds__(TH) void norm_backward_kernel(NormArgs a) {
    __shared__ double lds[2 * (TH / 64)];
    constexpr int GR = TH / R;   // rows at a time
    __shared__ __attribute__((aligned(16))) float sums[GR > 1 ? TH * V * 8 : 8];
    // w and dy in registers; the widest rows read them again, which come from L2
    constexpr bool kKeep = V == 1, kTiny = TH == kTinyThreads;
    const int lane = threadIdx.x % R;
    int turn_of = 0;
    float w[V][8], dw[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = (lane + v * R) * 8;
        if (kKeep)
            load_upto<float, 8>(a.w + c, a.D - c, w[v]);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            dw[v][i] = 0.0f;
    }
    const double mean = 1.0 / (double)a.D;
    const long long step = (long long)gridDim.x * GR;
    for (long long m0 = (long long)blockIdx.x * GR; m0 < a.M; m0 += step) {
        const long long mm = m0 + threadIdx.x / R;
        const bool live = mm < a.M;
        const long long m = live ? mm : a.M - 1;
        float r[V][8], g[V][8];
        const float *wr = a.w;
        asm volatile("" : "+s"(wr));   // read in every row, not once into registers
        double ss = 0.0, sg = 0.0;
        const F *rr = (const F *)a.res + m * a.sres;
        const E *dy = (const E *)a.x + m * a.sx;
        const F *dr = a.dr ? (const F *)a.dr + m * a.sdr : nullptr;
        // with two vectors a lane its registers are better left to a fourth wave a SIMD
        // (32768 x 1000 in bf16: 59 us, and 88 with the loads ahead)
        Raw8<F> td = {};
        if constexpr (kKeep) {
            const Raw8<F> tr = load8<kTiny>(rr, lane * 8, a.D);
            const Raw8<E> tg = load8<kTiny>(dy, lane * 8, a.D);
            if (dr)
                td = load8<kTiny>(dr, lane * 8, a.D);
            settle8<kTiny, F>(tr, lane * 8, a.D, r[0]);
            settle8<kTiny, E>(tg, lane * 8, a.D, g[0]);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = (lane + v * R) * 8;
                load_upto<F, 8>(rr + c, a.D - c, r[v]);
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (lane + v * R) * 8;
            if (!kKeep) {
                load_upto<float, 8>(wr + c, a.D - c, w[v]);
                load_upto<E, 8>(dy + c, a.D - c, g[v]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double rd = r[v][i];
                ss = __builtin_fma(rd, rd, ss);
                sg = __builtin_fma((double)w[v][i] * (double)g[v][i], rd, sg);
            }
        }
        ss = all_lanes64<Sum64, R>(ss, lds, turn_of);
        sg = all_lanes64<Sum64, R>(sg, lds, turn_of);
        const double var = __builtin_fma(ss, mean, a.eps);
        const double root = rsqrt64(var), k = -(sg * mean) * (root * root);
        const float inv = (float)root;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (lane + v * R) * 8;
            float o[8];
            if (kKeep && dr)
                settle8<kTiny, F>(td, c, a.D, o);
            else if (dr)
                load_upto<F, 8>(dr + c, a.D - c, o);
            if (!kKeep) {
                load_upto<float, 8>(wr + c, a.D - c, w[v]);
                load_upto<E, 8>(dy + c, a.D - c, g[v]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // converted again: the fp64 values of both passes at once would take
                // twice the registers
                asm volatile("" : "+v"(r[v][i]), "+v"(g[v][i]));
                if (live)
                    dw[v][i] = __builtin_fmaf(g[v][i] * inv, r[v][i], dw[v][i]);
                const float t =
                    inv * (float)__builtin_fma(k, (double)r[v][i],
                                               (double)w[v][i] * (double)g[v][i]);
                o[i] = dr ? o[i] + t : t;
            }
            if (live && a.r)
                store_upto<F, 8>((F *)a.r + m * a.sr + c, a.D - c, o);
            if (a.y) {
                if (a.drop.cut && c < a.D)
                    drop(a.drop, (unsigned long long)m * a.per + (lane + v * R), o);
                if (live)
                    store_upto<E, 8>((E *)a.y + m * a.sy + c, a.D - c, o);
            }
        }
    }
    float *part = a.partial + (long long)blockIdx.x * a.D;
    if (GR == 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (lane + v * R) * 8;
            store_upto<float, 8>(part + c, a.D - c, dw[v]);
        }
        return;
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
        store_vec<float, 8>(sums + ((threadIdx.x / R) * R * V + lane + v * R) * 8, dw[v]);
    __syncthreads();
    for (int c = threadIdx.x; c < a.D; c += TH) {
        float s = sums[c];
        for (int g = 1; g < GR; ++g)
            s += sums[g * (R * V * 8) + c];
        part[c] = s;
    }
}

// dw: the workgroups' sums, 32 groups of them in turn, then the groups in order (4 us for
// 1024 sums of 512).
__global__ __launch_bounds__(1024) void norm_sum_kernel(const float *partial, int parts, float *dw,
                                                        int D) {
    __shared__ float red[32][33];
    const int l = threadIdx.x & 31, g = threadIdx.x >> 5, c = blockIdx.x * 32 + l;
    float s = 0.0f;
    if (c < D)
        for (int p = g; p < parts; p += 256) {
            float v[8];   // in flight together
#pragma unroll
            for (int k = 0; k < 8; ++k)
                v[k] = partial[(long long)min(p + 32 * k, parts - 1) * D + c];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                s += p + 32 * k < parts ? v[k] : 0.0f;
        }
    red[g][l] = s;
    __syncthreads();
    if (g == 0 && c < D) {
        s = 0.0f;
        for (int i = 0; i < 32; ++i)
            s += red[i][l];
        dw[c] = s;
    }
}

// A thread eight elements, 16 bytes and one counter.  Bound by memory: 32768 x 2048 in
// bf16 with the residual 71 us, 403 MB at 5.6 TB/s (as above); the generator's 20 wide
// products an eight hide behind it.
template <typename E>
__global__ __launch_bounds__(256) void dropout_kernel(const E *x, long long sx, const E *res,
                                                      long long sr, E *y, long long sy, int M,
                                                      int D, int per, FastDiv div, Drop d) {
    const long long n = (long long)M * per;
    const long long step = (long long)gridDim.x * 256;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
        const int m = fdiv((int)i, div), c = ((int)i - m * per) * 8;
        float v[8], t[8];
        load_upto<E, 8>(x + m * sx + c, D - c, v);
        if (res)
            load_upto<E, 8>(res + m * sr + c, D - c, t);
        if (d.cut)
            drop(d, (unsigned long long)i, v);
        if (res)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v[j] += t[j];
        store_upto<E, 8>(y + m * sy + c, D - c, v);
    }
}

// ---- host ------------------------------------------------------------------------

inline int per_row(int D) { return D / 8 + (D % 8 != 0); }

inline bool make_drop(double p, unsigned long long seed, unsigned long long offset, Drop &d) {
    if (!(p >= 0.0 && p < 1.0))
        return false;
    const double cut = __builtin_rint(p * 65536.0);
    if (cut > 65535.0)
        return false;
    d.seed = seed;
    d.offset = offset;
    d.cut = (unsigned)cut;
    d.scale = (float)(65536.0 / (65536.0 - cut));
    return true;
}

inline bool norm_shape(int type, int rtype, int M, int D) {
    return type_size(type) && (rtype == type || rtype == FINC_F32) && M >= 0 && D >= 1 &&
           (long long)M * per_row(D) < (1ll << 31);
}

inline Region rows(const void *p, int M, long long s, int D, int size) {
    return {p, M, s, 1, 0, D, size};
}
// The alias that is taken: the same address, step and element size.
inline bool same(const Region &a, const Region &b) {
    return a.p == b.p && a.so == b.so && a.size == b.size;
}

enum { kForward, kFp8, kBackward };

// Calls f<E, F, R, V, TH>: lanes a row, vectors a lane and threads, by the width.  The
// forward holds little an element, so more vectors a lane spare it barriers.  The
// gradients hold three values an element and w and their sums in fp64, and the 8-bit
// output fp64 values: above 1024 one vector a lane, up to a whole workgroup a row
// (gradients of 32768 x 2048 in bf16: 115 us; 276 with four vectors in each lane of a
// wave a row, whose registers leave a wave a SIMD.  8 bits: 137 us and 185).  Up to
// 1024 a wave a row, two vectors a lane: with four waves a row a width just below fills
// two of them (32768 x 1000 in bf16: gradients 59 us and 103, 8 bits 56 and 130).
template <typename E, typename F, int KIND, typename Fn>
void with_width(int D, Fn fn) {
#define FINC_WIDTH(r, v, th)                                                              \
    return fn(E(), F(), std::integral_constant<int, r>(), std::integral_constant<int, v>(), \
              std::integral_constant<int, th>())
    if (D < 8)
        FINC_WIDTH(16, 1, kTinyThreads);
    if (D <= 128)
        FINC_WIDTH(16, 1, 256);
    if (D <= 512)
        FINC_WIDTH(64, 1, 256);
    if (D <= 1024)
        FINC_WIDTH(64, 2, 256);
    if constexpr (KIND != kForward) {
        if (D <= 2048)
            FINC_WIDTH(256, 1, 256);
        if (D <= 4096)
            FINC_WIDTH(512, 1, 512);
        if (D <= 8192)
            FINC_WIDTH(1024, 1, 1024);
    } else {
        if (D <= 2048)
            FINC_WIDTH(64, 4, 256);
        if (D <= 4096)
            FINC_WIDTH(256, 2, 256);
        if (D <= 8192)
            FINC_WIDTH(512, 2, 512);
    }
    FINC_WIDTH(1024, 2, 1024);
#undef FINC_WIDTH
}

// Workgroups that walk the rows of a gradient, a partial sum of dw each: four waves a
// SIMD, which the registers allow (32768 x 2048: 126 us, and 192 with half of them; 8192
// x 8192, whose workgroups are 16 waves: 127 us with 512 and 157 with 2048; 115 and 114
// since a row's loads are under way together).
inline int grad_blocks(int M, int D) {
    const long long blocks = cdivll(M > 0 ? M : 1, D <= 128 ? 16 : D <= 1024 ? 4 : 1);
    const long long most = D <= 2048 ? 1024 : 512;
    return (int)(blocks < most ? blocks : most);
}

template <int KIND, typename Fn>
void with_types(int type, int rtype, int D, Fn fn) {
    with_type(type, [&](auto e) {
        typedef decltype(e) E;
        if (rtype == type)
            with_width<E, E, KIND>(D, fn);
        else
            with_width<E, float, KIND>(D, fn);
    });
}

}  // namespace

extern "C" {

unsigned long long finc_dropout_counters(int M, int D) {
    return M < 0 || D < 1 ? 0 : (unsigned long long)M * per_row(D);
}

int finc_dropout(int type, const void *x, long long sx, const void *residual, long long sr,
                 void *y, long long sy, int M, int D, double p, unsigned long long seed,
                 unsigned long long offset, hipStream_t stream) {
    Drop d;
    if (!norm_shape(type, type, M, D) || !make_drop(p, seed, offset, d))
        return FINC_EINVAL;
    const int sz = type_size(type);
    const Region out = rows(y, M, sy, D, sz), rx = rows(x, M, sx, D, sz);
    const Region rr = rows(residual, residual ? M : 0, sr, D, sz);
    if (!readable(rx) || !readable(rr) || !writable(out) ||
        (overlap(out, rx) && !same(out, rx)) || (overlap(out, rr) && !same(out, rr)))
        return FINC_EINVAL;
    if (M == 0)
        return FINC_OK;
    const int per = per_row(D);
    with_type(type, [&](auto e) {
        typedef decltype(e) E;
        const long long blocks = cdivll((long long)M * per, 256);
        hipLaunchKernelGGL(dropout_kernel<E>, dim3((unsigned)(blocks < 16384 ? blocks : 16384)),
                           dim3(256), 0, stream, (const E *)x, sx, (const E *)residual, sr, (E *)y,
                           sy, M, D, per, make_fastdiv(per), d);
    });
    return launched();
}

int finc_add_norm_forward(const finc_norm_args *a, hipStream_t stream) {
    NormArgs c = {};
    if (!a || !norm_shape(a->type, a->rtype, a->M, a->D) || !(a->eps >= 0.0) ||
        !make_drop(a->p, a->seed, a->offset, c.drop))
        return FINC_EINVAL;
    if (a->D > FINC_MAX_ROW)
        return FINC_EUNSUPPORTED;
    const int sz = type_size(a->type), rz = type_size(a->rtype), M = a->M, D = a->D;
    const Region x = rows(a->x, M, a->sx, D, sz);
    const Region res = rows(a->residual, a->residual ? M : 0, a->sres, D, rz);
    const Region w = flat(a->w, D, 4);
    const Region y = rows(a->y, M, a->sy, D, a->scale ? 1 : sz);
    const Region r = rows(a->r, a->r ? M : 0, a->sr, D, rz);
    const Region s = flat(a->scale, a->scale ? M : 0, 4);
    if (!readable(x) || !readable(res) || !readable(w) || !writable(y) || !writable(r) ||
        !writable(s))
        return FINC_EINVAL;
    if ((overlap(y, x) && !same(y, x)) || overlap(y, res) || overlap(y, w) || overlap(y, r) ||
        overlap(y, s) || overlap(r, x) || (overlap(r, res) && !same(r, res)) || overlap(r, w) ||
        overlap(r, s) || overlap(s, x) || overlap(s, res) || overlap(s, w))
        return FINC_EINVAL;
    if (M == 0)
        return FINC_OK;
    c.x = a->x;
    c.res = a->residual;
    c.y = a->y;
    c.r = a->r;
    c.sx = a->sx;
    c.sres = a->sres;
    c.sy = a->sy;
    c.sr = a->sr;
    c.w = a->w;
    c.scale = a->scale;
    c.M = M;
    c.D = D;
    c.per = per_row(D);
    c.eps = a->eps;
    if (a->scale) {
        with_types<kFp8>(a->type, a->rtype, D, [&](auto e, auto f, auto R, auto V, auto TH) {
            const long long blocks = cdivll(M, TH / R), most = 8 * 256 * 256 / TH;
            hipLaunchKernelGGL((norm_fp8_kernel<decltype(e), decltype(f), R, V, TH>),
                               dim3((unsigned)(blocks < most ? blocks : most)), dim3(TH), 0,
                               stream, c);
        });
        return launched();
    }
    with_types<kForward>(a->type, a->rtype, D, [&](auto e, auto f, auto R, auto V, auto TH) {
        const long long blocks = cdivll(M, TH / R);
        const long long most = 8 * 256 * 256 / TH;   // eight waves a SIMD
        hipLaunchKernelGGL((norm_forward_kernel<decltype(e), decltype(f), R, V, TH>),
                           dim3((unsigned)(blocks < most ? blocks : most)), dim3(TH), 0, stream, c);
    });
    return launched();
}

size_t finc_add_norm_workspace_bytes(int M, int D) {
    if (!norm_shape(FINC_F32, FINC_F32, M, D) || D > FINC_MAX_ROW)
        return 0;
    return ((size_t)grad_blocks(M, D) * D * 4 + 255) / 256 * 256;
}

int finc_add_norm_backward(const finc_norm_grad_args *a, hipStream_t stream) {
    NormArgs c = {};
    if (!a || !norm_shape(a->type, a->rtype, a->M, a->D) || !(a->eps >= 0.0) ||
        !make_drop(a->p, a->seed, a->offset, c.drop) || ((uintptr_t)a->workspace & 255u))
        return FINC_EINVAL;
    if (a->D > FINC_MAX_ROW)
        return FINC_EUNSUPPORTED;
    const int sz = type_size(a->type), rz = type_size(a->rtype), M = a->M, D = a->D;
    const Region dy = rows(a->dy, M, a->sdy, D, sz), r = rows(a->r, M, a->sr, D, rz);
    const Region dr = rows(a->dr, a->dr ? M : 0, a->sdr, D, rz), w = flat(a->w, D, 4);
    const Region dx = rows(a->dx, a->dx ? M : 0, a->sdx, D, sz);
    const Region ds = rows(a->dresidual, a->dresidual ? M : 0, a->sdres, D, rz);
    const Region dw = flat(a->dw, D, 4);
    const Region ws = flat(a->workspace, (long long)finc_add_norm_workspace_bytes(M, D), 1);
    const Region in[] = {dy, r, dr, w}, out[] = {dx, ds, dw, ws};
    for (const Region &t : in)
        if (!readable(t))
            return FINC_EINVAL;
    for (const Region &t : out)
        if (!writable(t))
            return FINC_EINVAL;
    for (const Region &o : out)
        for (const Region &i : in)
            if (overlap(o, i) && !(&o == &out[0] && &i == &in[0] && same(o, i)) &&
                !(&o == &out[1] && &i == &in[2] && same(o, i)))
                return FINC_EINVAL;
    if (overlap(dx, ds) || overlap(dx, dw) || overlap(dx, ws) || overlap(ds, dw) ||
        overlap(ds, ws) || overlap(dw, ws))
        return FINC_EINVAL;
    c.x = a->dy;
    c.res = a->r;
    c.dr = a->dr;
    c.y = a->dx;
    c.r = a->dresidual;
    c.sx = a->sdy;
    c.sres = a->sr;
    c.sdr = a->sdr;
    c.sy = a->sdx;
    c.sr = a->sdres;
    c.w = a->w;
    c.partial = (float *)a->workspace;
    c.M = M;
    c.D = D;
    c.per = per_row(D);
    c.eps = a->eps;
    int parts = 0;
    if (M > 0) {
        parts = grad_blocks(M, D);
        with_types<kBackward>(a->type, a->rtype, D, [&](auto e, auto f, auto R, auto V, auto TH) {
            hipLaunchKernelGGL((norm_backward_kernel<decltype(e), decltype(f), R, V, TH>),
                               dim3((unsigned)parts), dim3(TH), 0, stream, c);
        });
        const int rc = launched();
        if (rc != FINC_OK)
            return rc;
    }
    hipLaunchKernelGGL(norm_sum_kernel, dim3((unsigned)cdivll(D, 32)), dim3(1024), 0, stream,
                       c.partial, parts, a->dw, D);
    return launched();
}

}  // extern "C"
