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
// The decay's follows from them: with S and dS before a part, and a' for a without what
// comes of the position's own pair of key and value,
//   dg_t = <S, dS> + sum_{s < t} (k_s . dk'_s - q_s . dq'_s).
// Every term passes a decay as dg does, so that it is as small where decays are strong: the
// own pair would cancel and leave its rounding (at a = -9 1% of dg, at -16 twenty times it),
// and so would a gradient of the last state in the same sums from the end.
// One kernel does all four, a role a tensor.
//
// A workgroup takes a part of up to 512 positions of one head, block by block, with S in
// its registers.  Longer rows have their parts' own sums formed first and joined by a scan,
// so that a single long row fills the card; which form is used follows from L alone.
//
// What bounds it: instructions.  One row of 16384 positions with 16 heads of 128 in bf16
// takes 144 us (45 the parts' sums, 18 their joining, 86 the rows), 268 MB, 52 us by memory;
// the vector ALU is busy 41% of the time and the matrix units 25%, with the two waves a SIMD
// that 256 registers a lane leave.
#include <type_traits>

#include "seq_mma.h"

namespace {

using namespace finc_seq;

constexpr int kBlock = 64;                       // positions of a block
constexpr int kPart = FINC_ATTENTION_PART;       // most positions of a workgroup
constexpr int kBlocks = kPart / kBlock;
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
    float *keep;            // of a single part: the state before it, 2 da dn apart
    float *last;            // of a single part: the state after it
    float *dots;            // (B H, L): dot . out, without the position's own pair
    int da, dn;             // elements of q and k, and of v
    int sd, sn;             // steps of a state's rows and columns
    float pscale, sscale, kscale;
    bool rev, out_f32;
    bool exact;             // the state may leave the call: its sums in full
};

struct Args {
    Role role[3];
    Tensor g;
    const float *decay;
    const int *lengths;
    float *local, *decays;   // states of the parts alone: (B H, parts + 1, da dn), (B H, parts)
    FastDiv by_bh, by_parts, by_h;
    int L, H, BH, parts, part, roles;   // positions of a part; roles of the launch
};

template <typename E>
__device__ inline const E *head_rows(const Tensor &t, int b, int h) {
    return (const E *)t.p + b * t.sb + (t.div == 1 ? h : h / t.div) * t.sh;
}

// ---- tiles in LDS --------------------------------------------------------------------
// 64 rows of D elements.  In 16 bits the 16-byte chunks of a row are exchanged by a
// function of the row, so that none of the reads below finds two of the lanes that go
// together in one bank: sixteen bytes of sixteen rows (sixteen lanes at a time: 0 to 3, 12
// to 15 and 20 to 27, the others of the first half, and so on), eight bytes of sixteen rows
// (32 lanes), and the transposed reads (32 lanes).

template <typename E, int D>
struct Rows {
    static constexpr int kLd = sizeof(E) == 2 ? D : D + 4;
    static constexpr int kSize = kBlock * kLd;
    __device__ static int turn(int r) {
        if constexpr (D == 128)
            return (r & 3) << 2 | (0x78 >> 2 * (r >> 2 & 3) & 3);
        else
            return (r & 2) | ((r >> 2 ^ r >> 3) & 1) << 2 | (r >> 3 & 1);
    }
    __device__ static int at(int r, int col) {
        if constexpr (sizeof(E) == 2)
            return r * kLd + ((col / 8 ^ turn(r)) * 8 | col % 8);
        else
            return r * kLd + col;
    }
    // A lane's places in the first rows and columns; those further on follow from them by
    // an exchange (a sum in 32 bits) that is formed where it is used: kept, they would take
    // some forty registers.
    struct Lane {
        int row, half, column, below;
    };
    __device__ static Lane lane(int l) {
        const int g = l >> 4, m = l & 15;
        const int r = sizeof(E) == 2 ? 8 * g + (m >> 2) : 8 * g;
        const int c = sizeof(E) == 2 ? 4 * (m & 3) : m;
        return {at(m, 8 * g), at(m, 4 * g), at(r, c), at(r + 4, c)};
    }
    __device__ static int there(int place, int r, int col) {   // multiples of 16
        return (sizeof(E) == 2 ? place ^ col : place + col) + r * kLd;
    }
    // Elements 8 g .. 8 g + 7 of the 32 from `col` on, of row r + m.
    __device__ static Frag<E> row(const E *s, const Lane &l, int r, int col) {
        return frag_row<E>(s + there(l.row, r, col));
    }
    // Elements 4 g .. 4 g + 3 of the 16 from `col` on, of row r + m.
    typedef E Four __attribute__((ext_vector_type(4)));
    __device__ static Four four(const E *s, const Lane &l, int r, int col) {
        return *(const Four *)(s + there(l.half, r, col));
    }
    // The same and those of the 16 behind them.
    __device__ static Frag<E> halves(const E *s, const Lane &l, int r, int col) {
        const Four a = four(s, l, r, col), b = four(s, l, r, col + 16);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    // Rows 8 g .. 8 g + 7 of the 32 from `r` on, of column col + m.
    __device__ static Frag<E> column(const E *s, const Lane &l, int r, int col) {
        if constexpr (sizeof(E) == 2) {
            const s16x4 a = read_transposed(s + there(l.column, r, col));
            const s16x4 b = read_transposed(s + there(l.below, r, col));
            return __builtin_bit_cast(Frag<E>,
                                      __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            Frag<E> v;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = s[there(l.column, r + i, col)];
            return v;
        }
    }
};

// A tile on its way there, sixteen bytes a thread and step.  The loads have no branches,
// which would wait for each: rows past the end are the last one, and the chunk that passes
// a row's end is the row's last sixteen bytes.  What that adds goes on the way to LDS.
template <typename E, int D, int THREADS>
struct Tile {
    static constexpr int V = kPer16<E>, kRow = D / V, kRows = THREADS / kRow;
    static constexpr int kSteps = kBlock / kRows;
    typedef typename Vec<E, V>::type Some;
    typedef E Whole __attribute__((ext_vector_type(V), aligned(16)));
    Some r[kSteps];

    // Rows of D elements whose steps stay within 31 bits of bytes over a tile.
    __device__ __attribute__((always_inline)) void load_whole(const E *p, int st, int rows) {
        const int col = (int)threadIdx.x % kRow * V, row = (int)threadIdx.x / kRow;
        const char *q = (const char *)p;
        if (rows >= kBlock) {
            const unsigned at = (row * st + col) * (unsigned)sizeof(E);
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
                r[i] = *(const Some *)(q + (long long)(i * kRows) * st * (int)sizeof(E) + at);
        } else {
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
                r[i] = *(const Some *)(q + (unsigned)((min(row + i * kRows, rows - 1) * st + col) *
                                                      (int)sizeof(E)));
        }
    }
    __device__ __attribute__((always_inline)) void load(const E *p, long long st, int rows,
                                                        int dim) {
        const int col = (int)threadIdx.x % kRow * V, row = (int)threadIdx.x / kRow;
        if (dim >= V) {
            const E *q = p + min(col, dim - V);
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
                r[i] = *(const Some *)(q + min(row + i * kRows, rows - 1) * st);
        } else {
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    r[i][j] = p[min(row + i * kRows, rows - 1) * st + min(j, dim - 1)];
        }
    }
    template <bool WHOLE>
    __device__ __attribute__((always_inline)) void store(E *s, int rows, int dim) const {
        const int col = (int)threadIdx.x % kRow * V, row = (int)threadIdx.x / kRow;
        // sixteen rows on, the chunks lie as they do here
        static_assert(sizeof(E) == 4 || kRows % 16 == 0, "one place a thread");
        E *to = s + Rows<E, D>::at(row, col);
        constexpr int kOn = kRows * Rows<E, D>::kLd;
        if constexpr (WHOLE) {
            if (rows >= kBlock) {
#pragma unroll
                for (int i = 0; i < kSteps; ++i)
                    *(Whole *)(to + i * kOn) = r[i];
            } else {
#pragma unroll
                for (int i = 0; i < kSteps; ++i)
                    *(Whole *)(to + i * kOn) = row + i * kRows < rows ? (Whole)r[i] : (Whole){};
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            typedef unsigned __int128 Bits;
            constexpr int kBits = 8 * (int)sizeof(E);
            Bits v = __builtin_bit_cast(Bits, (Whole)r[i]);
            if (dim % V != 0 && col + V > dim) {
                // where the load went back by as many elements, and the rest
                const int have = max(dim - col, 0);
                v = dim >= V ? v >> (kBits * min(V - have, V - 1)) : v;
                v = have > 0 ? v & (~(Bits)0 >> (kBits * (V - have))) : 0;
            }
            v = row + i * kRows < rows && col < dim ? v : 0;
            *(Whole *)(to + i * kOn) = __builtin_bit_cast(Whole, v);
        }
    }
};

// The weights of 64 queries and keys.
template <typename E>
struct Scores {
    typedef Rows<bf16, kBlock> R;
    bf16 hi[R::kSize], lo[R::kSize];
    // rows and columns from multiples of 16 on: four columns of row m
    __device__ void set(const typename R::Lane &l, int row, int col, f32x4 v) {
        bf16x4 a, b;
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
            float u[2] = {v[r], v[r + 1]};
            const bf16x2 h = part_of_two(u);
            const bf16x2 l = __builtin_convertvector((f32x2{u[0], u[1]}), bf16x2);
            a[r] = h[0], a[r + 1] = h[1];
            b[r] = l[0], b[r + 1] = l[1];
        }
        *(bf16x4 *)(hi + R::there(l.half, row, col)) = a;
        *(bf16x4 *)(lo + R::there(l.half, row, col)) = b;
    }
    __device__ Parts get(const typename R::Lane &l, int row, int col) const {
        return {R::row(hi, l, row, col), R::row(lo, l, row, col)};
    }
};
template <>
struct Scores<float> {
    typedef Rows<float, kBlock> R;
    float v[R::kSize];
    __device__ void set(const R::Lane &l, int row, int col, f32x4 x) {
        *(f32x4 *)(v + R::there(l.half, row, col)) = x;
    }
    __device__ f32x8 get(const R::Lane &l, int row, int col) const {
        return R::row(v, l, row, col);
    }
};
struct Nothing {
    typedef Rows<float, kBlock> R;
};

// Beside fp16 inputs a column of the state is held as 2^k times itself, its largest element
// in [2^13, 2^14), so that it goes into the products as two fp16 parts and the inputs as
// they are: two products where two bf16 parts of both took three, and the inputs' were
// formed by every wave (4 x 4096 x 16 heads of 128: 152 us, 264 before, and 399 for 656 of
// the gradients).  The power for `most`, the largest absolute value of this lane's part of
// a column that four lanes share.
__device__ inline int power(float most) {
    most = __builtin_fmaxf(most, __shfl_xor(most, 16));
    most = __builtin_fmaxf(most, __shfl_xor(most, 32));
    const int e = __builtin_bit_cast(int, most) >> 23;   // 255: infinite, which stays so
    return 13 + 127 - e;
}
// 2^k, |k| < 127
__device__ inline float two_to(int k) { return __builtin_bit_cast(float, (127 + k) << 23); }

// ---- the kernel ------------------------------------------------------------------

// STATES: the parts' own sums of k v^T alone, and their decays.
// DA, DN: elements of q and k, and of v, that the tiles hold.  A wave has 16 NC columns of
// v and of the state.  WHOLE: heads of DA and DN elements, steps of rows below 2^23 and
// outputs of the type; the code for all else next to it would take its registers.
constexpr int threads_of(int DN, int NC) { return 4 * DN / NC; }
// Tiles of columns of a wave: with two, what a wave reads of q and k serves twice as much
// (that bf16 prompt, again and again on the same inputs, 128 us, 145 with one).
constexpr int columns_of(int DN) { return DN / 64; }
template <typename E, int DA, int DN, int NC, bool STATES, bool WHOLE>
__global__ __launch_bounds__(threads_of(DN, NC), sizeof(E) == 2 ? 2 : 1)
    void attention_kernel(Args a) {
    typedef Mixed<E> M;
    typedef Rows<E, DA> R;
    typedef Rows<E, DN> RV;
    constexpr int WAVES = DN / 16 / NC;
    constexpr bool SCALED = std::is_same_v<E, f16>;   // the state's columns
    typedef Tile<E, DA, 64 * WAVES> T;
    typedef Tile<E, DN, 64 * WAVES> TV;
    __shared__ __align__(16) E sk[R::kSize];
    __shared__ __align__(16) E sv[RV::kSize];
    __shared__ __align__(16) E sq[STATES ? 8 : R::kSize];
    typedef std::conditional_t<STATES, Nothing, Scores<E>> P;
    __shared__ __align__(16) P sp;
    __shared__ __align__(16) float wk[kPart], ghi[kPart], glo[kPart], wq[kPart];
    __shared__ double total[kBlocks];
    __shared__ float sdot[WAVES][kBlock], own[kBlock];

    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int at = block_of();
    if (at >= a.BH * a.parts * (STATES ? 1 : a.roles))
        return;
    const int part = at - fdiv(at, a.by_parts) * a.parts;
    at = fdiv(at, a.by_parts);
    const int which = fdiv(at, a.by_bh), bh = at - which * a.BH;
    const int b = fdiv(bh, a.by_h), h = bh - b * a.H;
    const Role &o = a.role[which];
    const bool rev = o.rev;

    const int t0 = part * a.part;
    const int end = a.lengths ? min(max(a.lengths[b], 0), a.L) : a.L;
    const int have = min(max(end - t0, 0), a.part);            // valid positions
    const int blocks = (have + kBlock - 1) / kBlock;

    // Loads first, each behind the other: the first tiles, the state, the decays.
    // A state that leaves the call as fp32 takes its sums in full; for the outputs of 16
    // bits the two parts of its weights do.
    const bool exact = std::is_same_v<E, bf16> && (STATES || o.exact);
    const E *kp = head_rows<E>(o.k, b, h), *vp = head_rows<E>(o.v, b, h);
    const E *qp = STATES ? nullptr : head_rows<E>(o.q, b, h);
    T tk, tq;
    TV tv;
    auto fetch = [&](int c) __attribute__((always_inline)) {
        const long long t = t0 + c * kBlock;
        const int rows = have - c * kBlock;
        if constexpr (WHOLE) {
            tk.load_whole(kp + t * o.k.st, (int)o.k.st, rows);
            tv.load_whole(vp + t * o.v.st, (int)o.v.st, rows);
            if constexpr (!STATES)
                tq.load_whole(qp + t * o.q.st, (int)o.q.st, rows);
        } else {
            tk.load(kp + t * o.k.st, o.k.st, rows, o.da);
            tv.load(vp + t * o.v.st, o.v.st, rows, o.dn);
            if constexpr (!STATES)
                tq.load(qp + t * o.q.st, o.q.st, rows, o.da);
        }
    };
    if (blocks > 0)
        fetch(rev ? blocks - 1 : 0);

    // ---- the state ---------------------------------------------------------------
    // Element r of tile t is row 16 t + 4 g + r of column n: two tiles are the eight
    // elements that halves() gives of a query.
    const int n0 = 16 * NC * w;
    f32x4 S[DA / 16][NC];
    const long long size = (long long)o.da * o.dn;
    const float *init =
        !STATES && o.init ? o.init + bh * o.init_bh + part * o.init_p : nullptr;
#pragma unroll
    for (int t = 0; t < DA / 16; ++t)
#pragma unroll
        for (int c = 0; c < NC; ++c)
            S[t][c] = f32x4{0, 0, 0, 0};
    if (init) {
#pragma unroll
        for (int t = 0; t < DA / 16; ++t)
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if constexpr (WHOLE)
                        S[t][c][r] = init[(16 * t + r) * o.sd + 16 * c * o.sn +
                                          (unsigned)(4 * g * o.sd + (n0 + m) * o.sn)];
                    else
                        S[t][c][r] = init[min(16 * t + 4 * g + r, o.da - 1) * o.sd +
                                          min(n0 + 16 * c + m, o.dn - 1) * o.sn];
    }
    if (!STATES && o.keep)
        for (int i = threadIdx.x; i < size; i += 64 * WAVES)
            o.keep[bh * 2 * size + i] = init ? init[i] : 0.0f;

    // ---- the decays of the whole part: a wave a block ---------------------------
    const float base = a.decay ? a.decay[h] : 0.0f;
    const E *gp = a.g.p ? head_rows<E>(a.g, b, h) : nullptr;
    for (int c = w; c < blocks; c += WAVES) {
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

    if (!WHOLE && init) {
#pragma unroll
        for (int t = 0; t < DA / 16; ++t)
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    S[t][c][r] =
                        16 * t + 4 * g + r < o.da && n0 + 16 * c + m < o.dn ? S[t][c][r] : 0.0f;
    }

    // the tiles of scores that the products read but no block writes
    if constexpr (!STATES) {
        if (w < 2) {
            const int q = rev ? 2 * w + 1 : 2 * w, k = rev ? 2 * w : 2 * w + 1;
            sp.set(P::R::lane(lane), 16 * q, 16 * k, f32x4{0, 0, 0, 0});
        }
    }

    int k2[NC];   // the state is 2^-k2 times what is held (fp16)
#pragma unroll
    for (int e = 0; e < NC; ++e)
        k2[e] = init ? 0 : 126;
    auto rescale = [&]() __attribute__((always_inline)) {
        if constexpr (SCALED)
#pragma unroll
            for (int e = 0; e < NC; ++e) {
                float most = 0.0f;
#pragma unroll
                for (int t = 0; t < DA / 16; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        most = __builtin_fmaxf(most, __builtin_fabsf(S[t][e][r]));
                // a column of zeros has the largest power, below what is added to it next
                const int k = power(most) > 126 ? 126 - k2[e]
                                                : max(min(power(most), 126 - k2[e]), -126 - k2[e]);
                const float f = two_to(max(min(k, 126), -126));
                k2[e] += k;
#pragma unroll
                for (int t = 0; t < DA / 16; ++t)
                    S[t][e] *= f;
            }
    };
    if (init && blocks > 0)   // an empty row's state goes on as it is
        rescale();

    const typename R::Lane first = R::lane(lane);
    const typename RV::Lane first_v = RV::lane(lane);
    const typename P::R::Lane first_p = P::R::lane(lane);
    for (int i = 0; i < blocks; ++i) {
        const int c = rev ? blocks - 1 - i : i;
        const typename R::Lane l = {afresh(first.row), afresh(first.half), afresh(first.column),
                                    afresh(first.below)};
        const typename RV::Lane lv = {0, 0, DA == DN ? l.column : afresh(first_v.column),
                                      DA == DN ? l.below : afresh(first_v.below)};
        const typename P::R::Lane lp = {afresh(first_p.row), afresh(first_p.half), 0, 0};
        tk.template store<WHOLE>(sk, have - c * kBlock, o.da);
        tv.template store<WHOLE>(sv, have - c * kBlock, o.dn);
        if constexpr (!STATES)
            tq.template store<WHOLE>(sq, have - c * kBlock, o.da);
        __syncthreads();
        // asked for ahead of the next block's tiles, behind which a wait would be one for them
        typedef typename Vec<E, 4>::type Four;
        Four dot[4][NC];
        if (!STATES && o.dots) {
            const E *p = head_rows<E>(o.dot, b, h) + (t0 + c * kBlock) * o.dot.st;
            const int rows = have - c * kBlock;
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int e = 0; e < NC; ++e) {
                    const int row = min(16 * q + m, rows - 1), col = n0 + 16 * e + 4 * g;
                    if constexpr (WHOLE)
                        dot[q][e] = *(const Four *)((const char *)p + (unsigned)((row * (int)o.dot.st + col) * (int)sizeof(E)));
                    else if (o.dn % 4 == 0)
                        dot[q][e] = *(const Four *)(p + row * o.dot.st + min(col, o.dn - 4));
                    else
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            dot[q][e][r] = p[row * o.dot.st + min(col + r, o.dn - 1)];
                }
        }
        if (i + 1 < blocks)
            fetch(rev ? c - 1 : c + 1);

        if constexpr (!STATES) {
            // the scores' ten tiles that hold any, by their transposes
#pragma unroll 1   // their fragments take the registers of one at a time
            for (int i = 0; i < (10 + WAVES - 1) / WAVES; ++i) {
                const int tile = w + WAVES * i;
                if (tile < 10) {
                    const int big = (int)(0x3333222110ull >> 4 * tile) & 15;
                    const int small = (int)(0x3210210100ull >> 4 * tile) & 15;
                    const int qt = 16 * (rev ? small : big), kt = 16 * (rev ? big : small);
                    f32x4 p = {0, 0, 0, 0};
#pragma unroll
                    for (int d = 0; d < DA; d += 32)
                        p = mma(R::row(sk, l, kt, d), R::row(sq, l, qt, d), p);
                    const int qi = c * kBlock + qt + m, ki = c * kBlock + kt + 4 * g;
                    const float qh = ghi[qi], ql = glo[qi];
                    const f32x4 kh = *(const f32x4 *)(ghi + ki), kl = *(const f32x4 *)(glo + ki);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float e = (qh - kh[r]) + (ql - kl[r]);
                        e = __builtin_amdgcn_exp2f(rev ? -e : e) * o.pscale * p[r];
                        p[r] = (rev ? ki + r >= qi : ki + r <= qi) ? e : 0.0f;
                    }
                    if (o.dots && qt == kt) {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (ki + r == qi) {
                                own[qt + m] = p[r];
                                p[r] = 0.0f;
                            }
                    }
                    sp.set(lp, qt, kt, p);
                }
            }

            // the state's part, transposed: lane 16 g + m holds columns 4 g .. of row m
            f32x4 acc[4][NC];
#pragma unroll
            for (int d = 0; d < DA / 32; ++d) {
                __builtin_amdgcn_sched_barrier(0);
                typename M::Scaled st[NC];
#pragma unroll
                for (int e = 0; e < NC; ++e)
                    st[e] = M::scaled(__builtin_shufflevector(S[2 * d][e], S[2 * d + 1][e], 0, 1, 2,
                                                             3, 4, 5, 6, 7));
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const auto f = M::beside(R::halves(sq, l, 16 * q, 32 * d));
#pragma unroll
                    for (int e = 0; e < NC; ++e)
                        acc[q][e] = M::mma(st[e], f, d > 0 ? acc[q][e] : f32x4{0, 0, 0, 0});
                }
            }
            if constexpr (SCALED)
#pragma unroll
                for (int e = 0; e < NC; ++e) {
                    const float f = two_to(-k2[e]);
                    f32x4 of;
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        of[r] = __shfl(f, 4 * g + r);
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        acc[q][e] *= of;
                }
            __syncthreads();   // the scores
            typename M::Input v[2][NC];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < NC; ++e)
                    v[j][e] = M::input(RV::column(sv, lv, 32 * j, n0 + 16 * e));
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float u = wq[c * kBlock + 16 * q + m];
#pragma unroll
                for (int e = 0; e < NC; ++e)
                    acc[q][e] *= u;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (rev ? (j == 0 && q >= 2) : (j == 1 && q < 2))
                        continue;
                    const auto f = sp.get(lp, 16 * q, 32 * j);
#pragma unroll
                    for (int e = 0; e < NC; ++e)
                        acc[q][e] = M::mma(v[j][e], f, acc[q][e]);
                }
            }

            // ---- the rows' products with `dot`, then their own pairs, in fp32
            if (o.dots) {
                const typename RV::Lane here = {0, afresh(first_v.half), 0, 0};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float sum = 0.0f;
#pragma unroll
                    for (int e = 0; e < NC; ++e)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float u = acc[q][e][r] * (float)dot[q][e][r];
                            sum += WHOLE || n0 + 16 * e + 4 * g + r < o.dn ? u : 0.0f;
                        }
                    sum += __shfl_xor(sum, 16);
                    sum += __shfl_xor(sum, 32);
                    if (g == 0)
                        sdot[w][16 * q + m] = sum;
                    const float u = own[16 * q + m];
#pragma unroll
                    for (int e = 0; e < NC; ++e) {
                        const auto x = RV::four(sv, here, 16 * q, n0 + 16 * e);
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            acc[q][e][r] = __builtin_fmaf(u, (float)x[r], acc[q][e][r]);
                    }
                }
            }

            // ---- the rows
            const int rows = have - c * kBlock;   // past them: 0
            const long long row0 = b * o.ob + (t0 + c * kBlock) * o.ot + h * o.oh;
            if constexpr (WHOLE) {
                char *p = (char *)((E *)o.out + row0);
                const int size = (int)sizeof(E), stop = a.L - t0 - c * kBlock;
                const unsigned at = (m * (int)o.ot + n0 + 4 * g) * size;
                if (rows < kBlock)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int e = 0; e < NC; ++e)
                            acc[q][e] = 16 * q + m < rows ? acc[q][e] : f32x4{0, 0, 0, 0};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (16 * q + m < stop)
#pragma unroll
                        for (int e = 0; e < NC; ++e) {
                            float x[4];
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                x[r] = acc[q][e][r];
                            store_vec<E, 4>((E *)(p + (16ll * q * o.ot + 16 * e) * size + at), x);
                        }
                }
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int e = 0; e < NC; ++e) {
                        const int col = n0 + 16 * e + 4 * g, count = min(o.dn - col, 4);
                        const int t = 16 * q + m;
                        float x[4];
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            acc[q][e][r] = x[r] = t < rows ? acc[q][e][r] : 0.0f;
                        if (t0 + c * kBlock + t < a.L && count > 0) {
                            const long long i = row0 + t * o.ot + col;
                            if (o.out_f32)
                                store_upto<float, 4>((float *)o.out + i, count, x);
                            else
                                store_upto<E, 4>((E *)o.out + i, count, x);
                        }
                    }
            }
        }

        // ---- the state after the block
        const float f = __builtin_amdgcn_exp2f((float)total[c]);
        auto weigh = [&](int j, int e, f32x8 u) __attribute__((always_inline)) {
            return __builtin_convertvector(RV::column(sv, lv, 32 * j, n0 + 16 * e), f32x8) * u;
        };
        float by[NC];
        if constexpr (SCALED) {
#pragma unroll
            for (int e = 0; e < NC; ++e)
                by[e] = f * two_to(-k2[e]) * 0x1p14f;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const f32x8 u = frag_row<float>(wk + c * kBlock + 32 * j + 8 * g);
#pragma unroll
                for (int e = 0; e < NC; ++e) {
                    const f32x8 v = weigh(j, e, u);
#pragma unroll
                    for (int r = 0; r < 8; ++r)
                        by[e] = __builtin_fmaxf(by[e], __builtin_fabsf(v[r]));
                }
            }
#pragma unroll
            for (int e = 0; e < NC; ++e) {
                const int k = min(power(by[e]), 126);
                by[e] = two_to(k);
                const float decay = f * two_to(-k2[e]) * by[e];
                k2[e] = k;
#pragma unroll
                for (int t = 0; t < DA / 16; ++t)
                    S[t][e] *= decay;
            }
        } else {
#pragma unroll
            for (int t = 0; t < DA / 16; ++t)
#pragma unroll
                for (int e = 0; e < NC; ++e)
                    S[t][e] *= f;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const f32x8 u = frag_row<float>(wk + c * kBlock + 32 * j + 8 * g);
            f32x8 weighted[NC];
            typename M::Scaled v[NC];
#pragma unroll
            for (int e = 0; e < NC; ++e) {
                weighted[e] = weigh(j, e, u);
                if constexpr (SCALED)
                    weighted[e] *= by[e];
                v[e] = M::scaled(weighted[e]);
            }
            if constexpr (std::is_same_v<E, bf16>)
                if (exact) {
#pragma unroll
                    for (int e = 0; e < NC; ++e) {
                        bf16x8 rest;
                        v[e] = split(weighted[e], rest);
#pragma unroll
                        for (int t = 0; t < DA / 16; ++t)
                            S[t][e] = mma(R::column(sk, l, 32 * j, 16 * t), rest, S[t][e]);
                    }
                }
#pragma unroll
            for (int t = 0; t < DA / 16; ++t) {
                const auto k = M::beside(R::column(sk, l, 32 * j, 16 * t));
#pragma unroll
                for (int e = 0; e < NC; ++e)
                    S[t][e] = M::mma(k, v[e], S[t][e]);
            }
        }
        rescale();
        __syncthreads();
        if (!STATES && o.dots && w == 0) {
            const int t = c * kBlock + lane;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < WAVES; ++i)
                sum += sdot[i][lane];
            if (t < have)
                o.dots[(long long)bh * a.L + t0 + t] = sum;
        }
    }

    if constexpr (SCALED)
#pragma unroll
        for (int e = 0; e < NC; ++e)
#pragma unroll
            for (int t = 0; t < DA / 16; ++t)
                S[t][e] *= two_to(-k2[e]);

    // One of the two.  In a loop the addresses are formed here, not ahead of the blocks, where
    // they would spill five of heads' of 128 registers.
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
        ends[1] = o.last ? o.last + bh * size : nullptr;
    }
#pragma unroll 1
    for (int i = 0; i < 2; ++i) {
        float *p = i ? ends[1] : ends[0];
        if (!p)
            continue;
#pragma unroll
        for (int e = 0; e < NC; ++e) {
            const int n = n0 + 16 * e + m;
#pragma unroll
            for (int t = 0; t < DA / 16; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int d = 16 * t + 4 * g + r;
                    if (d < o.da && n < o.dn)
                        p[d * o.sd + n * o.sn] = S[t][e][r];
                }
        }
    }
    if constexpr (!STATES) {
        // rows past the length, behind the last block
        const int stop = min(a.L - t0, a.part);
        for (int t = blocks * kBlock + w; t < stop; t += WAVES)
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
                                                   int BH, int parts, int blocks, bool rev) {
    const int at = block_of(), bh = at / blocks;
    const int i = (at - bh * blocks) * 256 + (int)threadIdx.x;
    if (bh >= BH || i >= size)
        return;
    float *p = buf + bh * (long long)(parts + 1) * size + i;
    const float *d = decays + (long long)bh * parts;
    float s = first ? first[bh * (long long)size + i] : 0.0f;
    constexpr int kAhead = 8;
    for (int n0 = 0; n0 < parts; n0 += kAhead) {
        float l[kAhead];
#pragma unroll
        for (int n = 0; n < kAhead; ++n) {
            const int at = min(n0 + n, parts - 1), c = rev ? parts - 1 - at : at;
            l[n] = p[(long long)c * size];
        }
#pragma unroll
        for (int n = 0; n < kAhead; ++n)
            if (n0 + n < parts) {
                const int c = rev ? parts - 1 - (n0 + n) : n0 + n;
                p[(long long)c * size] = s;
                s = __builtin_fmaf(s, d[c], l[n]);
            }
    }
    p[(long long)parts * size] = s;
    if (last)
        last[bh * (long long)size + i] = s;
}

// dg of a part: what passes its start, and the sums from there on.  Log decays that count as
// the least one have no part in it: 0 there, not what the sums leave.
template <typename E>
__global__ __launch_bounds__(256) void decay_grad_kernel(
    const float *qdots, const float *kdots, const float *states, const float *grads, long long gbh,
    int first, Tensor g, const float *decay, E *dg, long long sb, long long st, long long sh,
    const int *lengths, int size, int BH, int L, int H, int parts, int span) {
    __shared__ double sums[256];
    const int at = block_of(), bh = at / parts, part = at - bh * parts;
    if (bh >= BH)
        return;
    const int b = bh / H, h = bh - b * H, tid = threadIdx.x;
    const int end = lengths ? min(max(lengths[b], 0), L) : L;
    // the state before the part and its gradient, the first part's at `first`
    const float *s = states + (bh * (long long)(parts + 1) + part) * size;
    const float *x = grads + bh * gbh + (part > 0 ? part - 1 : first) * (long long)size;
    // four sums of fp32 side by side, of 16 products each at most
    float some[4] = {0, 0, 0, 0};
    for (int i = 4 * tid; i < size; i += 1024) {
        float u[4], v[4];
        load_upto<float, 4>(s + i, size - i, u);
        load_upto<float, 4>(x + i, size - i, v);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            some[r] = __builtin_fmaf(u[r], v[r], some[r]);
    }
    sums[tid] = ((double)some[0] + some[1]) + ((double)some[2] + some[3]);
    __syncthreads();
    for (int d = 128; d > 0; d /= 2) {
        if (tid < d)
            sums[tid] += sums[tid + d];
        __syncthreads();
    }
    const double over = sums[0];
    __syncthreads();
    // the sums of the positions before t: two positions a thread
    const int t0 = part * span + 2 * tid;
    double v[2];
    for (int j = 0; j < 2; ++j) {
        const int t = t0 + j;
        const long long i = bh * (long long)L + t;
        v[j] = t < end && 2 * tid + j < span ? (double)kdots[i] - qdots[i] : 0.0;
    }
    sums[tid] = v[0] + v[1];
    __syncthreads();
    for (int d = 1; d < 256; d *= 2) {
        const double u = tid >= d ? sums[tid - d] : 0.0;
        __syncthreads();
        sums[tid] += u;
        __syncthreads();
    }
    const double before = tid > 0 ? sums[tid - 1] : 0.0;
    const E *gp = g.p ? head_rows<E>(g, b, h) : nullptr;
    const float base = decay ? decay[h] : 0.0f;
    for (int j = 0; j < 2; ++j) {
        const int t = t0 + j;
        if (t >= L || 2 * tid + j >= span)
            continue;
        float d = 0.0f;
        if (t < end && !(base + (gp ? (float)gp[t * g.st] : 0.0f) <= kLeast))   // NaN goes on
            d = (float)(over + before + (j ? v[0] : 0.0));
        dg[b * sb + t * st + h * sh] = (E)d;
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
    int B, S, H, DK, DV, cols;
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
    if (b >= a.B)
        return;
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

// Positions of a part, by the row's length alone, so that a row's bits do not depend on the
// batch: a short row's parts are halves, of which there are more side by side.  bf16, us with
// parts of 256 and of 512: one row of 2048 with 4 heads of 128 48 and 76, six of 1531 with 12 of
// 100 88 and 110; where rows fill the card, 64 with 16 heads of 128, 600 positions 481 and 532,
// 1024 681 and 590, 2048 1261 and 1066 (heads of 64: 171 and 209, 267 and 252, 472 and 459).
int part_of(int L) { return L > kPart && L <= 4 * kPart ? kPart / 2 : kPart; }
int parts_of(int L) { return L <= kPart ? 1 : (L - 1) / part_of(L) + 1; }
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

// Whether a role's heads fill their tiles, with steps that stay within 31 bits of bytes
// over a block.
bool fills(const Role &o, int size) {
    const long long far = (1ll << 31) / (kBlock * size);
    return (o.da == 64 || o.da == 128) && (o.dn == 64 || o.dn == 128) && !o.out_f32 && o.k.st < far &&
           o.v.st < far && (!o.out || (o.q.st < far && o.ot < far)) &&
           (!o.dots || o.dot.st < far);
}

// f with the type, the elements that the tiles hold and whether the heads fill them.
template <typename F>
void with_kernel(int type, const Role *o, int roles, F f) {
    bool whole = true;
    for (int i = 0; i < roles; ++i)
        whole = whole && fills(o[i], type_size(type));
    with_type(type, [&](auto e) {
        auto sized = [&](auto da, auto dn) {
            if (whole)
                f(e, da, dn, std::true_type());
            else
                f(e, da, dn, std::false_type());
        };
        const std::integral_constant<int, 64> half;
        const std::integral_constant<int, 128> full;
        if (o->da <= 64 && o->dn <= 64)
            sized(half, half);
        else if (o->da <= 64)
            sized(half, full);
        else if (o->dn <= 64)
            sized(full, half);
        else
            sized(full, full);
    });
}

// The parts' sums and the states between them.
void run_states(int type, Args &s, const float *first, float *last, hipStream_t stream) {
    const Role &o = s.role[0];
    with_kernel(type, &o, 1, [&](auto e, auto da, auto dn, auto whole) {
        constexpr int DA = decltype(da)::value, DN = decltype(dn)::value;
        constexpr int NC = columns_of(DN);
        attention_kernel<decltype(e), DA, DN, NC, true, decltype(whole)::value>
            <<<grid_of((long long)s.BH * s.parts), threads_of(DN, NC), 0, stream>>>(s);
    });
    const int size = o.da * o.dn, blocks = (size + 255) / 256;
    join_kernel<<<grid_of((long long)s.BH * blocks), 256, 0, stream>>>(
        s.local, s.decays, first, last, size, s.BH, s.parts, blocks, o.rev);
}

// Roles of one shape of tiles in one launch.
void run_roles(int type, Args s, int roles, hipStream_t stream) {
    while (roles > 0) {
        const Role &o = s.role[0];
        int n = 1;
        while (n < roles && (s.role[n].da > 64) == (o.da > 64) && (s.role[n].dn > 64) == (o.dn > 64))
            ++n;
        s.roles = n;
        with_kernel(type, &o, n, [&](auto e, auto da, auto dn, auto whole) {
            constexpr int DA = decltype(da)::value, DN = decltype(dn)::value;
            constexpr int NC = columns_of(DN);
            attention_kernel<decltype(e), DA, DN, NC, false, decltype(whole)::value>
                <<<grid_of((long long)s.BH * s.parts * n), threads_of(DN, NC), 0, stream>>>(s);
        });
        for (int i = n; i < roles; ++i)
            s.role[i - n] = s.role[i];
        roles -= n;
    }
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
    s.part = part_of(a->L);
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
        o.exact = true;
    }
    // rows of no position hand their state on: there is nothing to write but that
    if (L == 0 && !o.keep && !o.last)
        return FINC_OK;
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
    else
        n += round256((size_t)B * H * DK * DV * 4);   // the gradient of the state before them
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
        if (!g->dstate && dots)
            dstates = take((size_t)s.BH * size * 4);
        rv.last = g->dstate ? g->dstate : dstates;
        rv.exact = true;
    }
    if (L == 0 && !g->dstate)
        return FINC_OK;
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
                qdots, kdots, a->states, s.parts > 1 ? dstates : rv.last,
                s.parts > 1 ? (s.parts + 1) * size : size, s.parts > 1 ? s.parts : 0, s.g, a->decay,
                (E *)g->dg.p, g->dg.sb, g->dg.st, g->dg.sh, a->lengths, (int)size, s.BH, L, H,
                s.parts, s.part);
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
    s.B = B;
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
