// linear_attention.hip -- linear attention with a decay for each head and position: whole
// rows, their gradients, and one position (finc_linear_attention_* of finc.h).
//
// With G_t the sum of the log decays up to t, a block of 64 positions from the state S
// before it is three products on the matrix units:
//   y_i = sum_{j <= i} exp(G_i - G_j) (q_i . k_j) v_j + exp(G_i) q_i S,
//   S' = exp(G_end) S + sum_j exp(G_end - G_j) k_j v_j^T,
// in which every exponent is a difference of sums towards the later position, so that
// no factor passes 1 where the decays do not.  The gradients are the same form with
// other tensors in the places of q, k and v, two of them against the order:
//   dq: dy, v, k from S;   dk: v, dy, q and dv: k, q, dy from the state's gradient.
// The decay's follows from them: with <,> over all that lies behind t,
//   dg_t = sum_{s >= t} (q_s . dq_s - k_s . dk_s) + <S, dS>.
// One kernel does all four, a role a tensor.
//
// A workgroup takes a part of 512 positions of one head, block by block, with S in its
// registers.  Longer rows have their parts' own sums formed first and joined by a scan,
// so that a single long row fills the card; which form is used follows from L alone.
#include <type_traits>

#include "seq_mma.h"

namespace {

using namespace finc_seq;

constexpr int kBlock = 64;                       // positions of a block
constexpr int kPart = FINC_ATTENTION_PART;       // positions of a workgroup
constexpr int kBlocks = kPart / kBlock;
constexpr int kThreads = 256;
constexpr float kLeast = -128.0f;                // log decays below count as this

struct Tensor {
    const void *p;
    long long sb, st, sh;
    int div;   // heads that share a row
};

// What a workgroup computes: out of q, k and v, in the order of the positions or (rev)
// against it.
struct Role {
    Tensor q, k, v, dot;
    void *out;
    long long ob, ot, oh;
    const float *init;      // the state before each part, init_bh and init_p apart
    long long init_bh, init_p;
    float *keep;            // of a single part: the state before it and the one after it
    float *last;            // of a single part: the state after it
    float *dots;            // (B H, L): dot . out
    int da, dn;             // elements of q and k, and of v
    int sd, sn;             // steps of a state's rows and columns
    float pscale, sscale, kscale;
    bool rev, out_f32;
};

struct Args {
    Role role[3];
    Tensor g;
    const float *decay;
    const int *lengths;
    float *local, *decays;   // states of the parts alone: (B H, parts + 1, da dn), (B H, parts)
    FastDiv by_bh, by_parts, by_h;
    int L, H, BH, parts;
};

template <typename E>
__device__ inline const E *head_rows(const Tensor &t, int b, int h) {
    return (const E *)t.p + b * t.sb + (t.div == 1 ? h : h / t.div) * t.sh;
}

// ---- tiles on their way to LDS ---------------------------------------------------

// 64 rows of up to D elements, sixteen bytes a thread and step.
template <typename E, int D>
struct Tile {
    static constexpr int V = kPer16<E>, kRow = D / V, kRows = kThreads / kRow;
    static constexpr int kSteps = kBlock / kRows, kLd = D + V;
    typedef typename Vec<E, V>::type Some;
    Some r[kSteps];

    __device__ void load(const E *p, long long st, int rows, int dim) {
        const int col = (int)threadIdx.x % kRow * V, row = (int)threadIdx.x / kRow;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int at = row + i * kRows;
            Some v = {};
            if (at < rows && col < dim) {
                const E *q = p + at * st + col;
                if (col + V <= dim)
                    v = *(const Some *)q;
                else
                    for (int j = 0; j < V; ++j)
                        if (col + j < dim)
                            v[j] = q[j];
            }
            r[i] = v;
        }
    }
    __device__ void store(E *s) const {
        typedef E Whole __attribute__((ext_vector_type(V), aligned(16)));
        const int col = (int)threadIdx.x % kRow * V, row = (int)threadIdx.x / kRow;
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
            *(Whole *)(s + (row + i * kRows) * kLd + col) = r[i];
    }
};

// The weights of 64 queries and keys.
template <typename E>
struct Scores {
    static constexpr int kLd = kBlock + 8;
    bf16 hi[kBlock * kLd], lo[kBlock * kLd];
    __device__ void set(int row, int col, f32x4 v) {
        bf16x4 a, b;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            a[r] = (bf16)v[r];
            b[r] = (bf16)(v[r] - (float)a[r]);
        }
        *(bf16x4 *)(hi + row * kLd + col) = a;
        *(bf16x4 *)(lo + row * kLd + col) = b;
    }
    __device__ Parts get(int row, int col) const {
        return {frag_row<bf16>(hi + row * kLd + col), frag_row<bf16>(lo + row * kLd + col)};
    }
};
template <>
struct Scores<float> {
    static constexpr int kLd = kBlock + 4;
    float v[kBlock * kLd];
    __device__ void set(int row, int col, f32x4 x) { *(f32x4 *)(v + row * kLd + col) = x; }
    __device__ f32x8 get(int row, int col) const { return frag_row<float>(v + row * kLd + col); }
};

struct Nothing {};

// ---- the kernel ------------------------------------------------------------------

// STATES: the parts' own sums of k v^T alone, and their decays.
template <typename E, int D, bool STATES>
__global__ __launch_bounds__(kThreads, sizeof(E) == 2 ? 2 : 1) void attention_kernel(Args a) {
    typedef Mixed<E> M;
    typedef Tile<E, D> T;
    constexpr int LD = T::kLd, NC = D / 64;   // column tiles of a wave
    __shared__ __align__(16) E sk[kBlock * LD];
    __shared__ __align__(16) E sv[kBlock * LD];
    __shared__ __align__(16) E sq[STATES ? 8 : kBlock * LD];
    __shared__ __align__(16) std::conditional_t<STATES, Nothing, Scores<E>> sp;
    __shared__ __align__(16) float wk[kPart];
    __shared__ float ghi[kPart], glo[kPart], wq[kPart];
    __shared__ double total[kBlocks];
    __shared__ float sdot[4][kBlock];

    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int at = block_of();
    if (at >= a.BH * a.parts * (int)(STATES ? 1 : 3))   // the host gives whole roles
        return;
    const int part = at - fdiv(at, a.by_parts) * a.parts;
    at = fdiv(at, a.by_parts);
    const int which = fdiv(at, a.by_bh), bh = at - which * a.BH;
    const int b = fdiv(bh, a.by_h), h = bh - b * a.H;
    const Role &o = a.role[which];
    if (!STATES && !o.out)
        return;
    const bool rev = o.rev;

    const int t0 = part * kPart;
    const int end = a.lengths ? min(max(a.lengths[b], 0), a.L) : a.L;
    const int have = min(max(end - t0, 0), kPart);             // valid positions
    const int blocks = (have + kBlock - 1) / kBlock;

    // ---- the decays of the whole part: a wave a block ---------------------------
    const float base = a.decay ? a.decay[h] : 0.0f;
    const E *gp = a.g.p ? head_rows<E>(a.g, b, h) : nullptr;
    for (int c = w; c < blocks; c += 4) {
        const int t = c * kBlock + lane;
        float v = 0.0f;
        if (t < have) {
            v = base + (gp ? (float)gp[(t0 + t) * a.g.st] : 0.0f);
            v = v < kLeast ? kLeast : v;   // NaN stays
        }
        // in 64 bits, held as two floats: differences of neighbours keep their precision
        double s = v * 1.4426950408889634;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const double u = __shfl_up(s, d);
            s += lane >= d ? u : 0.0;
        }
        const double all = __shfl(s, 63);
        const float hi = (float)s;
        ghi[t] = hi;
        glo[t] = (float)(s - hi);
        const float from = __builtin_amdgcn_exp2f((float)s);
        const float to = __builtin_amdgcn_exp2f((float)(all - s));
        wq[t] = (rev ? to : from) * o.sscale;
        wk[t] = (rev ? from : to) * o.kscale;
        if (lane == 0)
            total[c] = all;
    }

    // ---- the state ---------------------------------------------------------------
    // Row 4 g + r of tile t is row d = 32 (t / 2) + 8 g + 4 (t % 2) + r, so that a lane's
    // values of two tiles are a fragment's eight neighbours.
    f32x4 S[D / 16][NC];
    const long long size = (long long)o.da * o.dn;
    const float *init =
        !STATES && o.init ? o.init + bh * o.init_bh + part * o.init_p : nullptr;
#pragma unroll
    for (int t = 0; t < D / 16; ++t)
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            S[t][c] = f32x4{0, 0, 0, 0};
            if (init) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int d = 32 * (t / 2) + 8 * g + 4 * (t % 2) + r;
                    const int n = 16 * (w * NC + c) + m;
                    const float v = init[min(d, o.da - 1) * o.sd + min(n, o.dn - 1) * o.sn];
                    S[t][c][r] = d < o.da && n < o.dn ? v : 0.0f;
                }
            }
        }
    if (!STATES && o.keep)
        for (int i = threadIdx.x; i < size; i += kThreads)
            o.keep[bh * 2 * size + i] = init ? init[i] : 0.0f;

    // the tiles of scores that the products read but no block writes
    if constexpr (!STATES) {
        if (w < 2) {
            const int q = rev ? 2 * w + 1 : 2 * w, k = rev ? 2 * w : 2 * w + 1;
            sp.set(16 * q + m, 16 * k + 4 * g, f32x4{0, 0, 0, 0});
        }
    }

    const E *kp = head_rows<E>(o.k, b, h), *vp = head_rows<E>(o.v, b, h);
    const E *qp = STATES ? nullptr : head_rows<E>(o.q, b, h);
    T tk, tv, tq;
    auto fetch = [&](int c) __attribute__((always_inline)) {
        const long long t = t0 + c * kBlock;
        const int rows = have - c * kBlock;
        tk.load(kp + t * o.k.st, o.k.st, rows, o.da);
        tv.load(vp + t * o.v.st, o.v.st, rows, o.dn);
        if constexpr (!STATES)
            tq.load(qp + t * o.q.st, o.q.st, rows, o.da);
    };
    if (blocks > 0)
        fetch(rev ? blocks - 1 : 0);

    for (int i = 0; i < blocks; ++i) {
        const int c = rev ? blocks - 1 - i : i;
        tk.store(sk);
        tv.store(sv);
        if constexpr (!STATES)
            tq.store(sq);
        __syncthreads();
        if (i + 1 < blocks)
            fetch(rev ? c - 1 : c + 1);

        // this wave's columns of v
        auto values = [&](int j, int n) __attribute__((always_inline)) {
            return frag_column<4>(sv + 32 * j * LD + 16 * (w * NC + n), LD, lane);
        };
        if constexpr (!STATES) {
            // the scores' ten tiles that hold any, by their transposes
#pragma unroll
            for (int n = 0; n < 3; ++n) {
                const int tile = w + 4 * n;
                if (tile < 10) {
                    const int big = (int)(0x3333222110ull >> 4 * tile) & 15;
                    const int small = (int)(0x3210210100ull >> 4 * tile) & 15;
                    const int qt = 16 * (rev ? small : big), kt = 16 * (rev ? big : small);
                    f32x4 p = {0, 0, 0, 0};
#pragma unroll
                    for (int s = 0; s < D; s += 32)
                        p = mma(frag_row<E>(sk + (kt + m) * LD + s + 8 * g),
                                frag_row<E>(sq + (qt + m) * LD + s + 8 * g), p);
                    const int qi = c * kBlock + qt + m, ki = c * kBlock + kt + 4 * g;
                    const float qh = ghi[qi], ql = glo[qi];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float e = (qh - ghi[ki + r]) + (ql - glo[ki + r]);
                        e = rev ? -e : e;
                        const bool in = rev ? ki + r >= qi : ki + r <= qi;
                        p[r] = in ? p[r] * (__builtin_amdgcn_exp2f(e) * o.pscale) : 0.0f;
                    }
                    sp.set(qt + m, kt + 4 * g, p);
                }
            }
        }

        f32x4 acc[4][NC];
        if constexpr (!STATES) {
            // the state's part, transposed: lane 16 g + m holds columns 4 g .. of row m
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int n = 0; n < NC; ++n)
                    acc[q][n] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                typename M::Value st[NC];
#pragma unroll
                for (int n = 0; n < NC; ++n)
                    st[n] = M::value(__builtin_shufflevector(S[2 * s][n], S[2 * s + 1][n], 0, 1, 2,
                                                             3, 4, 5, 6, 7));
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const auto f =
                        M::input(frag_row<E>(sq + (16 * q + m) * LD + 32 * s + 8 * g));
#pragma unroll
                    for (int n = 0; n < NC; ++n)
                        acc[q][n] = M::mma(st[n], f, acc[q][n]);
                }
            }
            __syncthreads();   // the scores
            typename M::Input v[2][NC];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int n = 0; n < NC; ++n)
                    v[j][n] = M::input(values(j, n));
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float u = wq[c * kBlock + 16 * q + m];
#pragma unroll
                for (int n = 0; n < NC; ++n)
                    acc[q][n] *= u;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (rev ? (j == 0 && q >= 2) : (j == 1 && q < 2))
                        continue;
                    const typename M::Value f = sp.get(16 * q + m, 32 * j + 8 * g);
#pragma unroll
                    for (int n = 0; n < NC; ++n)
                        acc[q][n] = M::mma(v[j][n], f, acc[q][n]);
                }
            }
        }

        if constexpr (!STATES) {
            // ---- the rows, and their products with `dot`
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int t = c * kBlock + 16 * q + m;
                const long long row = t0 + t;
                float sum = 0.0f;
#pragma unroll
                for (int n = 0; n < NC; ++n) {
                    const int col = 16 * (w * NC + n) + 4 * g, count = min(o.dn - col, 4);
                    float x[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        x[r] = t < have ? acc[q][n][r] : 0.0f;
                    if (row < a.L && count > 0) {
                        const long long i = b * o.ob + row * o.ot + h * o.oh + col;
                        if (o.out_f32)
                            store_upto<float, 4>((float *)o.out + i, count, x);
                        else
                            store_upto<E, 4>((E *)o.out + i, count, x);
                        if (o.dots && t < have) {
                            float y[4];
                            load_upto<E, 4>(head_rows<E>(o.dot, b, h) + row * o.dot.st + col, count,
                                            y);
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                sum = __builtin_fmaf(x[r], y[r], sum);
                        }
                    }
                }
                if (o.dots) {
                    sum += __shfl_xor(sum, 16);
                    sum += __shfl_xor(sum, 32);
                    if (g == 0)
                        sdot[w][16 * q + m] = sum;
                }
            }
        }

        // ---- the state after the block
        const float f = __builtin_amdgcn_exp2f((float)total[c]);
        typename M::Value vw[2][NC];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const f32x8 u = frag_row<float>(wk + c * kBlock + 32 * j + 8 * g);
#pragma unroll
            for (int n = 0; n < NC; ++n)
                vw[j][n] = M::value(__builtin_convertvector(values(j, n), f32x8) * u);
        }
#pragma unroll
        for (int t = 0; t < D / 16; ++t) {
#pragma unroll
            for (int n = 0; n < NC; ++n)
                S[t][n] *= f;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const auto k = M::input(frag_column<8>(
                    sk + 32 * j * LD + 32 * (t / 2) + 4 * (t % 2), LD, lane));
#pragma unroll
                for (int n = 0; n < NC; ++n)
                    S[t][n] = M::mma(k, vw[j][n], S[t][n]);
            }
        }

        __syncthreads();
        if (!STATES && o.dots && w == 0) {
            const int t = c * kBlock + lane;
            if (t < have)
                o.dots[(long long)bh * a.L + t0 + t] =
                    (sdot[0][lane] + sdot[1][lane]) + (sdot[2][lane] + sdot[3][lane]);
        }
    }

    float *ends[2] = {nullptr, nullptr};
    if constexpr (STATES) {
        ends[0] = a.local + (bh * (long long)(a.parts + 1) + part) * size;
        if (threadIdx.x == 0) {
            double s = 0.0;
            for (int c = 0; c < blocks; ++c)
                s += total[c];
            a.decays[(long long)bh * a.parts + part] = __builtin_amdgcn_exp2f((float)s);
        }
    } else {
        ends[0] = o.keep ? o.keep + (bh * 2 + 1) * size : nullptr;
        ends[1] = o.last ? o.last + bh * size : nullptr;
    }
#pragma unroll 1
    for (int i = 0; i < 2; ++i) {
        float *p = i ? ends[1] : ends[0];
        if (!p)
            continue;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int n = 16 * (w * NC + c) + m;
#pragma unroll
            for (int t = 0; t < D / 16; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int d = 32 * (t / 2) + 8 * g + 4 * (t % 2) + r;
                    if (d < o.da && n < o.dn)
                        p[d * o.sd + n * o.sn] = S[t][c][r];
                }
        }
    }
    if constexpr (!STATES) {
        // rows past the length, behind the last block
        const int stop = min(a.L - t0, kPart);
        for (int t = blocks * kBlock + w; t < stop; t += 4)
            for (int n = lane; n < o.dn; n += 64) {
                const long long i = b * o.ob + (t0 + t) * o.ot + h * o.oh + n;
                if (o.out_f32)
                    ((float *)o.out)[i] = 0.0f;
                else
                    ((E *)o.out)[i] = (E)0.0f;
            }
    }
}

// The states before every part and after the last one, from the parts' own sums (in
// place), or (rev) their gradients after every part and before the first one.
__global__ __launch_bounds__(256) void join_kernel(float *buf, const float *decays,
                                                   const float *first, float *last, int size,
                                                   int parts, int blocks, bool rev) {
    const int at = block_of(), bh = at / blocks;
    const int i = (at - bh * blocks) * 256 + (int)threadIdx.x;
    if (i >= size)
        return;
    float *p = buf + bh * (long long)(parts + 1) * size + i;
    float s = first ? first[bh * (long long)size + i] : 0.0f;
    for (int n = 0; n < parts; ++n) {
        const int c = rev ? parts - 1 - n : n;
        const float l = p[(long long)c * size];
        p[(long long)c * size] = s;
        s = __builtin_fmaf(s, decays[(long long)bh * parts + c], l);
    }
    p[(long long)parts * size] = s;
    if (last)
        last[bh * (long long)size + i] = s;
}

// dg of a part: the sums from its end, and what passes over its end.
template <typename E>
__global__ __launch_bounds__(256) void decay_grad_kernel(
    const float *qdots, const float *kdots, const float *states, const float *grads, long long gbh,
    const float *after, E *dg, long long sb, long long st, long long sh, const int *lengths,
    int size, int L, int H, int parts) {
    __shared__ double sums[256];
    const int at = block_of(), bh = at / parts, part = at - bh * parts;
    const int b = bh / H, h = bh - b * H, tid = threadIdx.x;
    const int end = lengths ? min(max(lengths[b], 0), L) : L;
    const float *s = states + (bh * (long long)(parts + 1) + part + 1) * size;
    const float *x = part + 1 < parts ? grads + bh * gbh + part * (long long)size
                                      : (after ? after + bh * (long long)size : nullptr);
    double over = 0.0;
    if (x)
        for (int i = tid; i < size; i += 256)
            over += (double)s[i] * x[i];
    sums[tid] = over;
    __syncthreads();
    for (int d = 128; d > 0; d /= 2) {
        if (tid < d)
            sums[tid] += sums[tid + d];
        __syncthreads();
    }
    over = sums[0];
    __syncthreads();
    // the sums from position t on: two positions a thread
    const int t0 = part * kPart + 2 * tid;
    double v[2];
    for (int j = 0; j < 2; ++j) {
        const int t = t0 + j;
        const long long i = bh * (long long)L + t;
        v[j] = t < end && 2 * tid + j < kPart ? (double)qdots[i] - kdots[i] : 0.0;
    }
    sums[tid] = v[0] + v[1];
    __syncthreads();
    for (int d = 1; d < 256; d *= 2) {
        const double u = tid + d < 256 ? sums[tid + d] : 0.0;
        __syncthreads();
        sums[tid] += u;
        __syncthreads();
    }
    const double behind = tid + 1 < 256 ? sums[tid + 1] : 0.0;
    for (int j = 0; j < 2; ++j) {
        const int t = t0 + j;
        if (t < L)
            dg[b * sb + t * st + h * sh] =
                (E)(t < end ? (float)(over + behind + (j ? v[1] : v[0] + v[1])) : 0.0f);
    }
}

// Gradients of shared heads: the sum of a group's, in order.
template <typename E>
__global__ __launch_bounds__(256) void group_sum_kernel(const float *part, E *out, long long sb,
                                                        long long st, long long sg, int L, int G,
                                                        int share, int D, long long rows) {
    const int vecs = (D + 3) / 4;
    const long long i = block_of() * 256ll + threadIdx.x;
    const long long row = i / vecs;   // of (B, L, G)
    if (row >= rows)
        return;
    const int col = (int)(i - row * vecs) * 4, count = min(D - col, 4);
    const long long bt = row / G, b = bt / L;
    const int gr = (int)(row - bt * G);
    const float *p = part + row * share * D + col;
    float s[4] = {0, 0, 0, 0};
    for (int h = 0; h < share; ++h) {
        float v[4];
        load_upto<float, 4>(p + (long long)h * D, count, v);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            s[r] += v[r];
    }
    store_upto<E, 4>(out + b * sb + (bt - b * L) * st + gr * sg + col, count, s);
}

// ---- one position ------------------------------------------------------------------

struct StepArgs {
    Tensor q, k, v, g;
    void *y;
    long long yb, yh;
    const float *decay;
    float *state;
    const int *slots;
    float scale;
    int S, H, DK, DV, cols;
    FastDiv by_cols, by_h;
};

// Bound by the state's way there and back.  A workgroup takes 32 columns of one head's
// state, four a lane and 32 rows side by side, so that few rows spread over many compute
// units; the rows' sums meet in registers and LDS in a fixed order.
template <typename E>
__global__ __launch_bounds__(256) void attention_step_kernel(StepArgs a) {
    __shared__ float part[4][8][4];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    int at = block_of();
    const int bh = fdiv(at, a.by_cols), block = at - bh * a.cols;
    const int b = fdiv(bh, a.by_h), h = bh - b * a.H;
    const int col = block * 32 + (lane & 7) * 4, count = a.DV - col;
    const int row = w * 8 + (lane >> 3);
    const int slot = a.slots ? a.slots[b] : b;
    E *y = (E *)a.y + b * a.yb + h * a.yh + col;
    if (slot < 0 || slot >= a.S) {
        const float zero[4] = {0, 0, 0, 0};
        if (row == 0)
            store_upto<E, 4>(y, min(count, 4), zero);
        return;
    }
    const E *q = head_rows<E>(a.q, b, h), *k = head_rows<E>(a.k, b, h);
    float l = a.decay ? a.decay[h] : 0.0f;
    if (a.g.p)
        l += (float)*head_rows<E>(a.g, b, h);
    l = l < kLeast ? kLeast : l;
    const float f = exp_fast(l);
    float v[4], s[FINC_MAX_HEAD / 32][4], sum[4] = {0, 0, 0, 0};
    float *p = a.state + ((long long)slot * a.H + h) * a.DK * a.DV + col;
#pragma unroll
    for (int i = 0; i < FINC_MAX_HEAD / 32; ++i) {
        const int d = row + 32 * i;
        load_upto<float, 4>(p + (long long)min(d, a.DK - 1) * a.DV, d < a.DK ? count : 0, s[i]);
    }
    load_upto<E, 4>(head_rows<E>(a.v, b, h) + col, count, v);
#pragma unroll
    for (int i = 0; i < FINC_MAX_HEAD / 32; ++i) {
        const int d = row + 32 * i;
        if (d < a.DK) {
            const float kd = (float)k[d], qd = (float)q[d];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[i][r] = __builtin_fmaf(f, s[i][r], kd * v[r]);
                sum[r] = __builtin_fmaf(qd, s[i][r], sum[r]);
            }
            store_upto<float, 4>(p + (long long)d * a.DV, min(count, 4), s[i]);
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        sum[r] += __shfl_xor(sum[r], 8);
        sum[r] += __shfl_xor(sum[r], 16);
        sum[r] += __shfl_xor(sum[r], 32);
        if (lane < 8)
            part[w][lane][r] = sum[r];
    }
    __syncthreads();
    if (tid < 8) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            sum[r] = a.scale * ((part[0][lane][r] + part[1][lane][r]) +
                                (part[2][lane][r] + part[3][lane][r]));
        store_upto<E, 4>(y, min(count, 4), sum);
    }
}

// ---- the host ------------------------------------------------------------------------

int parts_of(int L) { return L <= kPart ? 1 : (L + kPart - 1) / kPart; }
size_t round256(size_t n) { return (n + 255) / 256 * 256; }

bool attention_shape(int type, int B, int L, int H, int G, int DK, int DV) {
    return type_size(type) && B >= 0 && L >= 0 && H >= 1 && G >= 1 && H % G == 0 && DK >= 1 &&
           DK <= FINC_MAX_HEAD && DV >= 1 && DV <= FINC_MAX_HEAD &&
           (long long)B * H < (1ll << 24) && (long long)B * L < (1ll << 40) / ((long long)G * DK) &&
           (long long)B * L < (1ll << 40) / ((long long)H * DV) &&
           (long long)B * H * parts_of(L) < (1ll << 29);
}

// Element (b, t, h, d)'s region: an input may repeat, an output's elements must lie at
// different addresses.  As rows a step apart (and those between them) where they are, so
// that side by side views of one buffer are told apart; else as all that they span.
struct Heads {
    Region r;
    bool distinct;
};
Heads heads(const finc_heads &x, long long B, long long L, long long H, long long D, int size) {
    Heads o;
    o.distinct = false;
    if (B == 0 || L == 0) {
        o.r = flat(x.p, 0, size);
        o.distinct = true;
        return o;
    }
    long long n[3] = {B, L, H}, s[3] = {x.sb, x.st, x.sh};
    for (int i = 0; i < 3; ++i)
        if (s[i] < 0 || s[i] > (1ll << 57) / (n[i] > 1 ? n[i] : 1)) {
            o.r = {x.p, 2, -1, 1, 0, 1, size};   // no region
            return o;
        }
    const long long whole = (B - 1) * x.sb + (L - 1) * x.st + (H - 1) * x.sh + D;
    if (B == 1 || (x.st > 0 && x.sb % x.st == 0))
        o.r = {x.p, (B == 1 ? 0 : (B - 1) * (x.sb / x.st)) + L, x.st, H, x.sh, D, size};
    else if (L == 1)
        o.r = {x.p, B, x.sb, H, x.sh, D, size};
    else
        o.r = flat(x.p, whole, size);
    // from the smallest step on, each passes what lies below it
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (s[j] < s[i]) {
                const long long a = s[i], c = n[i];
                s[i] = s[j], n[i] = n[j];
                s[j] = a, n[j] = c;
            }
    long long below = D;
    o.distinct = true;
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1) {
            o.distinct = o.distinct && s[i] >= below;
            below += (n[i] - 1) * s[i];
        }
    return o;
}
bool good_out(const Heads &x) { return x.distinct && readable(x.r); }

Tensor tensor(const finc_heads &x, int div) { return {x.p, x.sb, x.st, x.sh, div}; }

// f with the type and the padded head dimension.
template <typename F>
void with_kernel(int type, int dim, F f) {
    with_type(type, [&](auto e) {
        if (dim <= 64)
            f(e, std::integral_constant<int, 64>());
        else
            f(e, std::integral_constant<int, 128>());
    });
}

// The parts' sums and the states between them.
void run_states(int type, Args &s, const float *first, float *last, hipStream_t stream) {
    const Role &o = s.role[0];
    with_kernel(type, o.da > o.dn ? o.da : o.dn, [&](auto e, auto d) {
        attention_kernel<decltype(e), decltype(d)::value, true>
            <<<grid_of((long long)s.BH * s.parts), kThreads, 0, stream>>>(s);
    });
    const int size = o.da * o.dn, blocks = (size + 255) / 256;
    join_kernel<<<grid_of((long long)s.BH * blocks), 256, 0, stream>>>(
        s.local, s.decays, first, last, size, s.parts, blocks, o.rev);
}

void run_roles(int type, const Args &s, int roles, hipStream_t stream) {
    const Role &o = s.role[0];
    with_kernel(type, o.da > o.dn ? o.da : o.dn, [&](auto e, auto d) {
        attention_kernel<decltype(e), decltype(d)::value, false>
            <<<grid_of((long long)s.BH * s.parts * roles), kThreads, 0, stream>>>(s);
    });
}

Args common(const finc_attention_args *a) {
    Args s = {};
    s.g = tensor(a->g, 1);
    s.decay = a->decay;
    s.lengths = a->lengths;
    s.L = a->L;
    s.H = a->H;
    s.BH = a->B * a->H;
    s.parts = parts_of(a->L);
    s.by_bh = make_fastdiv(s.BH);
    s.by_parts = make_fastdiv(s.parts);
    s.by_h = make_fastdiv(s.H);
    return s;
}

}  // namespace

extern "C" {

size_t finc_linear_attention_states_bytes(int B, int L, int H, int DK, int DV) {
    if (!attention_shape(FINC_F32, B, L, H, 1, DK, DV))
        return 0;
    const size_t parts = parts_of(L), bh = (size_t)B * H;
    return round256(bh * (parts + 1) * DK * DV * 4) + round256(bh * parts * 4);
}

int finc_linear_attention_forward(const finc_attention_args *a, hipStream_t stream) {
    if (!a || !attention_shape(a->type, a->B, a->L, a->H, a->G, a->DK, a->DV) ||
        ((uintptr_t)a->states & 255u))
        return FINC_EINVAL;
    const int sz = type_size(a->type), B = a->B, L = a->L, H = a->H, G = a->G;
    const long long st = (long long)B * H * a->DK * a->DV;
    const size_t keep = finc_linear_attention_states_bytes(B, L, H, a->DK, a->DV);
    const Heads y = heads(a->y, B, L, H, a->DV, sz);
    const Region in[] = {heads(a->q, B, L, G, a->DK, sz).r, heads(a->k, B, L, G, a->DK, sz).r,
                         heads(a->v, B, L, H, a->DV, sz).r,
                         a->g.p ? heads(a->g, B, L, H, 1, sz).r : flat(nullptr, 0, sz),
                         flat(a->decay, a->decay ? H : 0, 4),
                         flat(a->lengths, a->lengths ? B : 0, 4),
                         flat(a->state != a->state_out ? a->state : nullptr,
                              a->state && a->state != a->state_out ? st : 0, 4)};
    const Region out[] = {y.r, flat(a->state_out, a->state_out ? st : 0, 4),
                          flat(a->states, a->states ? (long long)keep : 0, 1)};
    for (const Region &r : in)
        if (!readable(r))
            return FINC_EINVAL;
    for (const Region &r : out)
        if (!readable(r))
            return FINC_EINVAL;
    if (!good_out(y) || !disjoint(in, out))
        return FINC_EINVAL;
    if (B == 0)
        return FINC_OK;
    Args s = common(a);
    if (s.parts > 1 && !a->states)
        return FINC_EINVAL;
    Role &o = s.role[0];
    o.q = tensor(a->q, H / G);
    o.k = tensor(a->k, H / G);
    o.v = tensor(a->v, 1);
    o.out = a->y.p;
    o.ob = a->y.sb;
    o.ot = a->y.st;
    o.oh = a->y.sh;
    o.da = a->DK;
    o.dn = a->DV;
    o.sd = a->DV;
    o.sn = 1;
    o.pscale = o.sscale = (float)a->scale;
    o.kscale = 1.0f;
    const long long size = (long long)a->DK * a->DV;
    if (s.parts > 1) {
        s.local = a->states;
        s.decays = (float *)((char *)a->states +
                             round256((size_t)s.BH * (s.parts + 1) * size * 4));
        run_states(a->type, s, a->state, a->state_out, stream);
        o.init = a->states;
        o.init_bh = (s.parts + 1) * size;
        o.init_p = size;
    } else {
        o.init = a->state;
        o.init_bh = size;
        o.keep = a->states;
        o.last = a->state_out;
    }
    // rows of no position hand their state on: there is nothing to write but that
    if (L == 0 && !o.keep && !o.last)
        return FINC_OK;
    if (L == 0 && !o.out)
        o.out = (void *)(o.keep ? o.keep : o.last);   // not written: no row
    run_roles(a->type, s, 1, stream);
    return launched();
}

size_t finc_linear_attention_workspace_bytes(int B, int L, int H, int G, int DK, int DV) {
    if (!attention_shape(FINC_F32, B, L, H, G, DK, DV))
        return 0;
    const size_t bl = (size_t)B * L * H;
    size_t n = 2 * round256(bl * 4);   // the rows' products for dg
    if (parts_of(L) > 1)
        n += finc_linear_attention_states_bytes(B, L, H, DK, DV);
    if (G < H)
        n += 2 * round256(bl * DK * 4);
    return n;
}

int finc_linear_attention_backward(const finc_attention_args *a, const finc_attention_grads *g,
                                   hipStream_t stream) {
    if (!a || !g || !attention_shape(a->type, a->B, a->L, a->H, a->G, a->DK, a->DV) ||
        ((uintptr_t)a->states & 255u) || ((uintptr_t)g->workspace & 255u))
        return FINC_EINVAL;
    const int sz = type_size(a->type), B = a->B, L = a->L, H = a->H, G = a->G, DK = a->DK,
              DV = a->DV;
    const long long size = (long long)DK * DV, st = B * (long long)H * size;
    const size_t keep = finc_linear_attention_states_bytes(B, L, H, DK, DV);
    const size_t space = finc_linear_attention_workspace_bytes(B, L, H, G, DK, DV);
    const Heads dq = heads(g->dq, B, L, G, DK, sz), dk = heads(g->dk, B, L, G, DK, sz),
                dv = heads(g->dv, B, L, H, DV, sz);
    Heads dg = {flat(nullptr, 0, sz), true};
    if (g->dg.p)
        dg = heads(g->dg, B, L, H, 1, sz);
    const Region in[] = {heads(a->q, B, L, G, DK, sz).r, heads(a->k, B, L, G, DK, sz).r,
                         heads(a->v, B, L, H, DV, sz).r, heads(g->dy, B, L, H, DV, sz).r,
                         a->g.p ? heads(a->g, B, L, H, 1, sz).r : flat(nullptr, 0, sz),
                         flat(a->decay, a->decay ? H : 0, 4),
                         flat(a->lengths, a->lengths ? B : 0, 4),
                         flat(a->states, (long long)keep, 1),
                         flat(g->dstate_out, g->dstate_out ? st : 0, 4)};
    const Region out[] = {dq.r, dk.r, dv.r, dg.r, flat(g->dstate, g->dstate ? st : 0, 4),
                          flat(g->workspace, (long long)space, 1)};
    for (const Region &r : in)
        if (!readable(r))
            return FINC_EINVAL;
    for (const Region &r : out)
        if (!readable(r))
            return FINC_EINVAL;
    if (!good_out(dq) || !good_out(dk) || !good_out(dv) || !good_out(dg) || !disjoint(in, out))
        return FINC_EINVAL;
    if (B == 0)
        return FINC_OK;
    Args s = common(a);
    char *ws = (char *)g->workspace;
    auto take = [&](size_t bytes) {
        char *p = ws;
        ws += round256(bytes);
        return (float *)p;
    };
    const size_t bl = (size_t)B * L * H;
    float *qdots = take(bl * 4), *kdots = take(bl * 4);
    float *parts_q = nullptr, *parts_k = nullptr, *dstates = nullptr;
    if (G < H) {
        parts_q = take(bl * DK * 4);
        parts_k = take(bl * DK * 4);
    }
    const bool dots = g->dg.p != nullptr;
    const Tensor q = tensor(a->q, H / G), k = tensor(a->k, H / G), v = tensor(a->v, 1),
                 dy = tensor(g->dy, 1);
    const float scale = (float)a->scale;

    Role &rv = s.role[0], &rk = s.role[1], &rq = s.role[2];
    rv.q = k;
    rv.k = q;
    rv.v = dy;
    rv.out = g->dv.p;
    rv.ob = g->dv.sb;
    rv.ot = g->dv.st;
    rv.oh = g->dv.sh;
    rv.da = DK;
    rv.dn = DV;
    rv.sd = DV;
    rv.sn = 1;
    rv.rev = true;
    rv.pscale = rv.kscale = scale;
    rv.sscale = 1.0f;
    rk = rv;
    rk.q = v;
    rk.k = dy;
    rk.v = q;
    rk.da = DV;
    rk.dn = DK;
    rk.sd = 1;
    rk.sn = DV;
    rq = rk;
    rq.rev = false;
    rq.q = dy;
    rq.k = v;
    rq.v = k;
    rq.pscale = rq.sscale = scale;
    rq.kscale = 1.0f;
    auto shared = [&](Role &o, const finc_heads &x, float *part) {
        o.out = part ? part : x.p;
        o.out_f32 = part != nullptr;
        o.ob = part ? (long long)L * H * DK : x.sb;
        o.ot = part ? (long long)H * DK : x.st;
        o.oh = part ? DK : x.sh;
    };
    shared(rk, g->dk, parts_k);
    shared(rq, g->dq, parts_q);
    if (dots) {
        rk.dot = k;
        rk.dots = kdots;
        rq.dot = q;
        rq.dots = qdots;
    }
    rq.init = a->states;
    rq.init_bh = (s.parts + 1) * size;
    rq.init_p = size;
    if (s.parts > 1) {
        dstates = take((size_t)s.BH * (s.parts + 1) * size * 4);
        s.local = dstates;
        s.decays = take((size_t)s.BH * s.parts * 4);
        run_states(a->type, s, g->dstate_out, g->dstate, stream);
        rv.init = rk.init = dstates;
        rv.init_bh = rk.init_bh = (s.parts + 1) * size;
        rv.init_p = rk.init_p = size;
    } else {
        rv.init = rk.init = g->dstate_out;
        rv.init_bh = rk.init_bh = size;
        rv.last = g->dstate;
    }
    if (L == 0 && !g->dstate)
        return FINC_OK;
    if (L == 0 && !rv.out)
        rv.out = g->dstate;   // not written: no row
    run_roles(a->type, s, L == 0 ? 1 : 3, stream);
    if (L == 0)
        return launched();
    with_type(a->type, [&](auto e) {
        typedef decltype(e) E;
        if (G < H) {
            const long long rows = (long long)B * L * G, vecs = (DK + 3) / 4;
            const dim3 grid = grid_of(cdivll(rows * vecs, 256));
            group_sum_kernel<E><<<grid, 256, 0, stream>>>(parts_q, (E *)g->dq.p, g->dq.sb, g->dq.st,
                                                          g->dq.sh, L, G, H / G, DK, rows);
            group_sum_kernel<E><<<grid, 256, 0, stream>>>(parts_k, (E *)g->dk.p, g->dk.sb, g->dk.st,
                                                          g->dk.sh, L, G, H / G, DK, rows);
        }
        if (dots)
            decay_grad_kernel<E><<<grid_of((long long)s.BH * s.parts), 256, 0, stream>>>(
                qdots, kdots, a->states, dstates, (s.parts + 1) * size, g->dstate_out,
                (E *)g->dg.p, g->dg.sb, g->dg.st, g->dg.sh, a->lengths, (int)size, L, H, s.parts);
    });
    return launched();
}

int finc_linear_attention_step(const finc_attention_step_args *a, hipStream_t stream) {
    if (!a || a->S < 0 || !attention_shape(a->type, a->B, 1, a->H, a->G, a->DK, a->DV) ||
        (!a->slots && a->S < a->B))
        return FINC_EINVAL;
    const int sz = type_size(a->type), B = a->B, H = a->H, G = a->G, DK = a->DK, DV = a->DV;
    const Heads y = heads(a->y, B, 1, H, DV, sz);
    const Region in[] = {heads(a->q, B, 1, G, DK, sz).r, heads(a->k, B, 1, G, DK, sz).r,
                         heads(a->v, B, 1, H, DV, sz).r,
                         a->g.p ? heads(a->g, B, 1, H, 1, sz).r : flat(nullptr, 0, sz),
                         flat(a->decay, a->decay ? H : 0, 4), flat(a->slots, a->slots ? B : 0, 4)};
    const Region out[] = {y.r, flat(a->state, elements(a->S, (long long)H * DK, DV), 4)};
    for (const Region &r : in)
        if (!readable(r))
            return FINC_EINVAL;
    for (const Region &r : out)
        if (!readable(r))
            return FINC_EINVAL;
    if (!good_out(y) || !disjoint(in, out))
        return FINC_EINVAL;
    if (B == 0)
        return FINC_OK;
    StepArgs s = {};
    s.q = tensor(a->q, H / G);
    s.k = tensor(a->k, H / G);
    s.v = tensor(a->v, 1);
    s.g = tensor(a->g, 1);
    s.y = a->y.p;
    s.yb = a->y.sb;
    s.yh = a->y.sh;
    s.decay = a->decay;
    s.state = a->state;
    s.slots = a->slots;
    s.scale = (float)a->scale;
    s.S = a->S;
    s.H = H;
    s.DK = DK;
    s.DV = DV;
    s.cols = (DV + 31) / 32;
    s.by_cols = make_fastdiv(s.cols);
    s.by_h = make_fastdiv(H);
    with_type(a->type, [&](auto e) {
        attention_step_kernel<decltype(e)>
            <<<grid_of((long long)B * H * s.cols), 256, 0, stream>>>(s);
    });
    return launched();
}

}  // extern "C"
