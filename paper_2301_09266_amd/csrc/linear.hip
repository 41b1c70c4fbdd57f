// linear.hip -- projections of rows with bias, activation and residual, and their
// gradients (finc_linear_* of finc.h).
//
// Three products: y = x w^T (both operands lie along the sum), dx = d w (w lies across
// it) and dw = d^T x (both do).  An operand that lies across the sum is transposed on
// its way from LDS to the matrix units, so that no transposed copy is made.
#include <math.h>

#include <type_traits>

#include "seq_mma.h"

namespace {

using namespace finc_seq;

constexpr int kThreads = 256;

// ---- activations -----------------------------------------------------------------

// The normal distribution's function and density.  Below 0 the function is exp(-p^2 / 2)
// times a smooth function of |p| that falls as 1 / |p|: t P(t) with t = 1 / (1 + |p| / 4), P a
// fit of degree 9 (relative error 4e-8), so that far negative p keep its relative precision
// (1e-6 of it; the exponent's rounding is added back).  32768 x 1024 x 4096 with GELU: 444 us
// with erfcf, 367 so, 268 without.
struct Normal {
    float cdf, density;
};
__device__ inline Normal normal(float p) {
    const float x = __builtin_fminf(__builtin_fabsf(p), 1e15f);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.25f, x, 1.0f));
    float r = 0.019782036376224436f;
    r = __builtin_fmaf(r, t, -0.08087742544062713f);
    r = __builtin_fmaf(r, t, 0.09559727708714869f);
    r = __builtin_fmaf(r, t, -0.03171769001371136f);
    r = __builtin_fmaf(r, t, 0.0636991908558743f);
    r = __builtin_fmaf(r, t, 0.05897512916000919f);
    r = __builtin_fmaf(r, t, 0.08160311151676858f);
    r = __builtin_fmaf(r, t, 0.09346635515367649f);
    r = __builtin_fmaf(r, t, 0.09973643161775542f);
    r = __builtin_fmaf(r, t, 0.09973556672301861f);
    // exp(-x^2 / 2) = 2^(h + rest), in which rest is what h and its factors round away
    constexpr float L = -0.7213475108146667f, kRest = -9.629815e-09f;
    const float q = x * x, h = q * L;
    float rest = __builtin_fmaf(q, L, -h);
    rest = __builtin_fmaf(q, kRest, rest);
    rest = __builtin_fmaf(__builtin_fmaf(x, x, -q), L, rest);
    const float e = __builtin_amdgcn_exp2f(h);
    const float f = __builtin_fmaf(e * 0.69314718055994531f, x < 64.0f ? rest : 0.0f, e);
    const float low = f * (r * t), cdf = p < 0.0f ? low : 1.0f - low;
    return {p == p ? cdf : p, 0.39894228040143268f * f};
}
__device__ inline float act_value(int act, float p) {
    switch (act) {
    case FINC_ACT_RELU:
        return p < 0.0f ? 0.0f : p;   // NaN stays
    case FINC_ACT_SILU:
        return silu(p);
    case FINC_ACT_GELU:
        return __builtin_fmaxf(p, -1e30f) * normal(p).cdf;
    default:
        return p;
    }
}
__device__ inline float act_grad(int act, float p) {
    switch (act) {
    case FINC_ACT_RELU:
        return p > 0.0f ? 1.0f : (p <= 0.0f ? 0.0f : p);
    case FINC_ACT_SILU:
        return silu_grad(p, sigmoid(p));
    default: {
        const Normal n = normal(p);
        return __builtin_fmaf(__builtin_amdgcn_fmed3f(p, -1e15f, 1e15f), n.density, n.cdf);
    }
    }
}

// ---- the product -------------------------------------------------------------------
// C (M, N) = sum over K of A and B.  An operand (rows, K) along the sum has its rows `s`
// apart; across it, (K, rows), its positions of the sum.

struct Gemm {
    const void *a, *b;
    long long sa, sb;
    void *c;                  // of the type, or fp32 partial sums (split > 1)
    long long sc;
    const float *bias;
    const void *residual;
    long long sr;
    void *pre;
    long long sp;
    int M, N, K, act, split, per;   // positions of the sum a split has
    int tiles_m, tiles_n;
};

// Bias, what the gradients keep, activation and residual of N neighbouring columns.
template <typename E, int N>
__device__ __attribute__((always_inline)) inline void finish(const Gemm &o, long long row, int col,
                                                             int count, float (&v)[N]) {
    if (o.bias) {
        float u[N];
        load_upto<float, N>(o.bias + col, count, u);
#pragma unroll
        for (int r = 0; r < N; ++r)
            v[r] += u[r];
    }
    if (o.pre)
        store_upto<E, N>((E *)o.pre + row * o.sp + col, count, v);
#pragma unroll
    for (int r = 0; r < N; ++r)
        v[r] = act_value(o.act, v[r]);
    if (o.residual) {
        float u[N];
        load_upto<E, N>((const E *)o.residual + row * o.sr + col, count, u);
#pragma unroll
        for (int r = 0; r < N; ++r)
            v[r] += u[r];
    }
}

// One operand's tile: ROWS rows by BK positions of the sum, sixteen bytes a thread and
// step.  ACROSS: BK rows of LDS of ROWS elements.
template <typename E, int ROWS, int BK, bool ACROSS>
struct Operand {
    static constexpr int V = kPer16<E>, kOuter = ACROSS ? BK : ROWS, kInner = ACROSS ? ROWS : BK;
    static constexpr int kRow = kInner / V, kRows = kThreads / kRow, kSteps = kOuter / kRows;
    static constexpr int kLd = kInner + V;
    typedef typename Vec<E, V>::type Some;
    Some r[kSteps];

    // from (row0, k0) on, of `rows` rows and the sum's positions below k1
    __device__ __attribute__((always_inline)) void load(const E *p, long long s, int row0, int rows,
                                                        int k0, int k1) {
        const int in = (int)threadIdx.x % kRow * V, out = (int)threadIdx.x / kRow;
        const int o0 = ACROSS ? k0 : row0, o1 = ACROSS ? k1 : rows;
        const int i0 = ACROSS ? row0 : k0, i1 = ACROSS ? rows : k1;
        const int count = i1 - i0 - in;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int at = o0 + out + i * kRows;
            Some v = {};
            if (at < o1 && count > 0) {
                const E *q = p + at * s + i0 + in;
                if (count >= V)
                    v = *(const Some *)q;
                else {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const E e = q[min(j, count - 1)];
                        v[j] = j < count ? e : (E)0.0f;
                    }
                }
            }
            r[i] = v;
        }
    }
    __device__ __attribute__((always_inline)) void store(E *s) const {
        typedef E Whole __attribute__((ext_vector_type(V), aligned(16)));
        const int in = (int)threadIdx.x % kRow * V, out = (int)threadIdx.x / kRow;
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
            *(Whole *)(s + (out + i * kRows) * kLd + in) = r[i];
    }
    // rows row .. row + 15, positions k .. k + 31 of the sum
    __device__ __attribute__((always_inline)) static Frag<E> frag(const E *s, int row, int k,
                                                                  int lane) {
        if constexpr (ACROSS)
            return frag_column<4>(s + k * kLd + row, kLd, lane);
        else
            return frag_row<E>(s + (row + (lane & 15)) * kLd + k + 8 * (lane >> 4));
    }
};

// Four waves, two by two.  Lanes hold four neighbouring columns of a row of C.
template <typename E, int BM, int BN>
struct AnyTile {
    static constexpr int BK = 128 / sizeof(E);
    // either operand along the sum or across it
    static constexpr int kBytes =
        (Operand<E, BM, BK, false>::kOuter * Operand<E, BM, BK, false>::kLd >
                 Operand<E, BM, BK, true>::kOuter * Operand<E, BM, BK, true>::kLd
             ? Operand<E, BM, BK, false>::kOuter * Operand<E, BM, BK, false>::kLd
             : Operand<E, BM, BK, true>::kOuter * Operand<E, BM, BK, true>::kLd) *
        (int)sizeof(E);
    static_assert(BM == BN, "both operands' places");
};
template <typename E, int BM, int BN, bool AA, bool BA>
__device__ __attribute__((always_inline)) inline void gemm_any(const Gemm &o, int at, char *lds) {
    constexpr int BK = 128 / sizeof(E), TM = BM / 32, TN = BN / 32;
    typedef Operand<E, BM, BK, AA> OA;
    typedef Operand<E, BN, BK, BA> OB;
    E *sa = (E *)lds, *sb = (E *)(lds + AnyTile<E, BM, BN>::kBytes);
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles = o.tiles_m * o.tiles_n;
    const int part = at / tiles;
    at -= part * tiles;
    if (part >= o.split)
        return;
    const int m0 = at / o.tiles_n * BM, n0 = at % o.tiles_n * BN;
    const int k0 = part * o.per, k1 = min(k0 + o.per, o.K);
    const int wm = (w >> 1) * (BM / 2), wn = (w & 1) * (BN / 2);

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
            acc[i][j] = f32x4{0, 0, 0, 0};
    OA a;
    OB b;
    a.load((const E *)o.a, o.sa, m0, o.M, k0, k1);
    b.load((const E *)o.b, o.sb, n0, o.N, k0, k1);
    for (int k = k0; k < k1; k += BK) {
        a.store(sa);
        b.store(sb);
        __syncthreads();
        if (k + BK < k1) {
            a.load((const E *)o.a, o.sa, m0, o.M, k + BK, k1);
            b.load((const E *)o.b, o.sb, n0, o.N, k + BK, k1);
        }
#pragma unroll
        for (int s = 0; s < BK; s += 32) {
            Frag<E> fa[TM], fb[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i)
                fa[i] = OA::frag(sa, wm + 16 * i, s, lane);
#pragma unroll
            for (int j = 0; j < TN; ++j)
                fb[j] = OB::frag(sb, wn + 16 * j, s, lane);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = mma(fb[j], fa[i], acc[i][j]);
        }
        __syncthreads();
    }

#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int row = m0 + wm + 16 * i + m;
        if (row >= o.M)
            continue;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int col = n0 + wn + 16 * j + 4 * g, count = min(o.N - col, 4);
            if (count <= 0)
                continue;
            float v[4];
#pragma unroll
            for (int r = 0; r < 4; ++r)
                v[r] = acc[i][j][r];
            if (o.split > 1) {
                store_upto<float, 4>((float *)o.c + ((long long)part * o.M + row) * o.N + col,
                                     count, v);
                continue;
            }
            finish<E, 4>(o, row, col, count, v);
            store_upto<E, 4>((E *)o.c + row * o.sc + col, count, v);
        }
    }
}

template <typename E, int BM, int BN, bool AA, bool BA>
__global__ __launch_bounds__(kThreads) void gemm_kernel(Gemm o) {
    __shared__ __align__(16) char lds[2 * AnyTile<E, BM, BN>::kBytes];
    gemm_any<E, BM, BN, AA, BA>(o, block_of(), lds);
}

// ---- the product of aligned operands -------------------------------------------------
// Tiles go from memory to LDS without registers between, 16 bytes a lane, a few stages of
// 32 positions ahead; fragments are read a stage ahead of their products.  The 16-byte
// chunks of a stage's rows are exchanged by a function of the row so that the lanes of a
// read, which take the same chunk of sixteen rows, find them in different banks.
// Positions and rows past the ends come from sixteen zero bytes.

constexpr int kStep = 32;   // positions of the sum of a stage

__device__ __align__(16) const float kZeros[4] = {0, 0, 0, 0};

// Waits until at most N of this wave's loads are under way, and for the other waves.
template <int N>
__device__ __attribute__((always_inline)) inline void arrive() {
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <typename E, int ROWS, int WAVES, bool ACROSS>
struct Stage {
    static constexpr int V = kPer16<E>, BK = kStep;
    static constexpr int kLd = ACROSS ? ROWS : BK;                // elements of an LDS row
    static constexpr int kChunks = kLd / V;                       // chunks of one
    static constexpr int kBytes = ROWS * BK * (int)sizeof(E);
    static constexpr int kLoads = kBytes / 1024 / WAVES;          // of a wave

    // What a chunk's place is exchanged with in row `r`.  Reads of 16 bytes go by sixteen
    // lanes: 0 to 3, 12 to 15 and 20 to 27, the others of the first half, and so on.
    __device__ static int turn(int r) {
        const int f = 0x78 >> 2 * (r >> 3 & 3) & 3;   // 0, 2, 3, 1
        if constexpr (!ACROSS && sizeof(E) == 2)
            return f;
        else if constexpr (!ACROSS)
            return (r >> 1 & 1) | f << 1;
        else if constexpr (sizeof(E) == 2)   // units of two chunks
            return ((r & 3) | (r >> 3 & 3) << 2) << 1 & (kChunks - 1);
        else                                 // units of four
            return (r >> 3 & 3) << 2;
    }

    const E *p[kLoads];   // this lane's places of the next stage
    int at[kLoads];       // their positions of the sum
    long long step;

    // Rows past the operand's end are its last ones: what comes of them is not stored.
    __device__ __attribute__((always_inline)) void start(const E *base, long long s, int row0,
                                                         int rows, int k0, int wave, int lane) {
        step = ACROSS ? BK * s : BK;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int chunk = (wave * kLoads + i) * 64 + lane;
            const int r = chunk / kChunks;
            const int c = (chunk % kChunks ^ turn(r)) * V;
            if constexpr (ACROSS) {
                at[i] = k0 + r;
                p[i] = base + at[i] * s + min(row0 + c, rows - V);
            } else {
                at[i] = k0 + c;
                p[i] = base + min(row0 + r, rows - 1) * s + at[i];
            }
        }
    }
    __device__ __attribute__((always_inline)) void load(char *lds, int k1, int wave) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const void *from = at[i] < k1 ? (const void *)p[i] : (const void *)kZeros;
            __builtin_amdgcn_global_load_lds(
                (const __attribute__((address_space(1))) void *)from,
                (__attribute__((address_space(3))) void *)(lds + (wave * kLoads + i) * 1024), 16, 0,
                0);
            p[i] += step;
            at[i] += BK;
        }
    }
    // Row (of the operand) of index i of tile t of a wave.  Along the sum two tiles take
    // eight neighbouring rows in turns, so that a lane's results are eight neighbours.
    __device__ static int row(int t, int i) {
        return ACROSS ? 16 * t + i : 32 * (t / 2) + 8 * (i / 4) + 4 * (t % 2) + i % 4;
    }
    // Where a lane's part of tile 0 of the rows from row0 on lies in a stage.  row0 is a
    // multiple of 32 (along) or of the rows of a wave, a power of two (across): what a tile
    // adds to that, frag() gives the reads as an offset, or exchanges the place with.
    __device__ static int place(int row0, int lane) {
        const int g = lane >> 4, m = lane & 15;
        int at;
        if constexpr (!ACROSS) {
            const int r = row0 + row(0, m);
            at = r * kLd + ((sizeof(E) == 2 ? g : 2 * g) ^ turn(r)) * V;
        } else {
            const int r = 8 * g + (sizeof(E) == 2 ? m >> 2 : 0);
            const int col = row0 + (sizeof(E) == 2 ? 4 * (m & 3) : m);
            at = r * kLd + ((col / V) ^ turn(r)) * V + col % V;
        }
        return at * (int)sizeof(E);
    }
    __device__ __attribute__((always_inline)) static Frag<E> frag(const char *lds, int place,
                                                                  int t) {
        if constexpr (!ACROSS) {
            const int more = (32 * (t / 2) + 4 * (t % 2)) * kLd * (int)sizeof(E);
            if constexpr (sizeof(E) == 2)
                return frag_row<E>((const E *)(lds + place + more));
            else {
                typedef float F4 __attribute__((ext_vector_type(4)));
                const F4 a = *(const F4 *)(lds + place + more);
                const F4 b = *(const F4 *)(lds + (place ^ 16) + more);
                return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
            }
        } else if constexpr (sizeof(E) == 2) {
            const E *q = (const E *)(lds + (place ^ 16 * t * (int)sizeof(E)));
            const s16x4 a = read_transposed(q), b = read_transposed(q + 4 * kLd);
            return __builtin_bit_cast(Frag<E>,
                                      __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const E *q = (const E *)(lds + (place ^ 16 * t * (int)sizeof(E)));
            Frag<E> v;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = q[i * kLd];
            return v;
        }
    }
};

// Where a lane's results lie: `row0` and `col0` are its wave's first.
template <typename SA, typename SB>
struct Place {
    int row0, col0, lane;
    __device__ long long row(int i) const { return row0 + SA::row(i, lane & 15); }
    __device__ int col(int j) const { return col0 + SB::row(j, 4 * (lane >> 4)); }
};

// From the sums to the outputs, a tile's rows after each other.  WHOLE: no column lies past
// the end.  PLAIN: a gradient's, whose columns are whole chunks and which has no epilogue.
// A wait for a load is one for the stores before it: the bias is there beforehand, and four
// rows' residuals are asked for together.
template <typename E, bool WHOLE, bool PLAIN, typename P, int TM, int TN>
__device__ __attribute__((always_inline)) inline void emit(const Gemm &o, int part, const P &at,
                                                           f32x4 (&acc)[TM][TN]) {
    constexpr int N = PLAIN ? 4 : 8, J = TN * 4 / N;   // neighbouring columns, and their sets
    constexpr int A = TM < 4 ? TM : 4;
    typedef typename Vec<E, N>::type Some;
    auto put = [&](auto *p, long long row, long long step, const float *v)
                   __attribute__((always_inline)) {
        typedef std::remove_reference_t<decltype(*p)> T;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int col = at.col(j * (N / 4));
            if constexpr (WHOLE || PLAIN) {
                if (WHOLE || col < o.N)
                    store_vec<T, N>(p + row * step + col, v + j * N);
            } else
                store_upto<T, N>(p + row * step + col, o.N - col, v + j * N);
        }
    };
    float bias[J * N] = {};
    if (!PLAIN && o.bias && o.split == 1) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int col = at.col(j * (N / 4));
            load_upto<float, N>(o.bias + col, WHOLE ? N : o.N - col, bias + j * N);
        }
    }
#pragma unroll
    for (int i0 = 0; i0 < TM; i0 += A) {
        Some res[A][J];
        if (!PLAIN && o.residual && o.split == 1) {
#pragma unroll
            for (int i = 0; i < A; ++i)
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const int col = at.col(j * (N / 4)), count = o.N - col;
                    const long long row = min(at.row(i0 + i), (long long)o.M - 1);
                    const E *p = (const E *)o.residual + row * o.sr + col;
                    if constexpr (WHOLE)
                        res[i][j] = *(const Some *)p;
                    else if (count > 0)
#pragma unroll
                        for (int r = 0; r < N; ++r)
                            res[i][j][r] = p[min(r, count - 1)];
                }
        }
#pragma unroll
        for (int i = 0; i < A; ++i) {
            const long long row = at.row(i0 + i);
            if (row >= o.M)
                continue;
            float v[J * N];
#pragma unroll
            for (int r = 0; r < J * N; ++r)
                v[r] = acc[i0 + i][r / 4][r % 4];
            if (o.split > 1) {
                put((float *)o.c + part * (long long)o.M * o.N, row, o.N, v);
                continue;
            }
            if constexpr (!PLAIN) {
#pragma unroll
                for (int r = 0; r < J * N; ++r)
                    v[r] += bias[r];
                if (o.pre)
                    put((E *)o.pre, row, o.sp, v);
                auto apply = [&](auto act) __attribute__((always_inline)) {
#pragma unroll
                    for (int r = 0; r < J * N; ++r)
                        v[r] = act_value(decltype(act)::value, v[r]);
                };
                if (o.act == FINC_ACT_RELU)
                    apply(std::integral_constant<int, FINC_ACT_RELU>());
                else if (o.act == FINC_ACT_SILU)
                    apply(std::integral_constant<int, FINC_ACT_SILU>());
                else if (o.act == FINC_ACT_GELU)
                    apply(std::integral_constant<int, FINC_ACT_GELU>());
                if (o.residual)
#pragma unroll
                    for (int r = 0; r < J * N; ++r)
                        v[r] += (float)res[i][r / N][r % N];
            }
            put((E *)o.c, row, o.sc, v);
        }
    }
}

template <typename E, int BM, int BN, int WM, int WN, int STAGES, bool AA, bool BA>
__device__ __attribute__((always_inline)) inline void gemm_fast(
    const Gemm &o, int at, char (*lds)[(BM + BN) * kStep * (int)sizeof(E)]) {
    typedef Stage<E, BM, WM * WN, AA> SA;
    typedef Stage<E, BN, WM * WN, BA> SB;
    constexpr int BK = kStep, TM = BM / WM / 16, TN = BN / WN / 16;
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // Blocks go to the eight dies in turns: each die takes neighbouring tiles, in groups of
    // eight rows of tiles that are walked column by column, so that its cache holds both.
    const int tiles = o.tiles_m * o.tiles_n;
    const int part = at / tiles;
    if (part >= o.split)
        return;
    at -= part * tiles;
    {
        const int die = at & 7, each = tiles / 8, more = tiles & 7;
        at = die * each + min(die, more) + (at >> 3);
        const int band = 8 * o.tiles_n, first = at / band * 8, rows = min(8, o.tiles_m - first);
        const int in = at - first * o.tiles_n;
        at = (first + in % rows) * o.tiles_n + in / rows;
    }
    const int m0 = at / o.tiles_n * BM, n0 = at % o.tiles_n * BN;
    const int k0 = part * o.per, k1 = min(k0 + o.per, o.K);
    const int wm = w / WN * (BM / WM), wn = w % WN * (BN / WN);

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
            acc[i][j] = f32x4{0, 0, 0, 0};
    SA a;
    SB b;
    a.start((const E *)o.a, o.sa, m0, o.M, k0, w, lane);
    b.start((const E *)o.b, o.sb, n0, o.N, k0, w, lane);
    const int steps = (k1 - k0 + BK - 1) / BK;
    // Stage s + STAGES - 1 is asked for while the fragments of stage s + 1 are read and
    // those of stage s multiplied.  Past the last one zeros are, so that the counts hold.
    constexpr int kLoads = SA::kLoads + SB::kLoads;
    int to = 0;
    auto ask = [&]() __attribute__((always_inline)) {
        a.load(lds[to], k1, w);
        b.load(lds[to] + SA::kBytes, k1, w);
        to = to + 1 == STAGES ? 0 : to + 1;
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s)
        ask();
    // The first half of a stage's rows and its columns are read while the second half of
    // the stage before is multiplied, the second half while the first one is.
    constexpr int H = TM / 2;
    Frag<E> fa[H], fc[H], fb[TN], fd[TN];
    const int pa = SA::place(wm, lane), pb = SB::place(wn, lane);
    int from = 0;
    auto first = [&](Frag<E>(&rb)[TN]) __attribute__((always_inline)) {
        const char *la = lds[from], *lb = la + SA::kBytes;
#pragma unroll
        for (int j = 0; j < TN; ++j)
            rb[j] = SB::frag(lb, pb, j);
#pragma unroll
        for (int i = 0; i < H; ++i)
            fa[i] = SA::frag(la, pa, i);
    };
    auto second = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < H; ++i)
            fc[i] = SA::frag(lds[from], pa, H + i);
        from = from + 1 == STAGES ? 0 : from + 1;
    };
    auto step = [&](Frag<E>(&now)[TN], Frag<E>(&next)[TN]) __attribute__((always_inline)) {
        ask();
        second();
#pragma unroll
        for (int i = 0; i < H; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
                acc[i][j] = mma(now[j], fa[i], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
        first(next);
#pragma unroll
        for (int i = 0; i < H; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
                acc[H + i][j] = mma(now[j], fc[i], acc[H + i][j]);
        __builtin_amdgcn_sched_barrier(0);
        arrive<kLoads *(STAGES - 3)>();
    };
    arrive<kLoads *(STAGES - 2)>();
    first(fb);
    arrive<kLoads *(STAGES - 3)>();
    for (int s = 0; s < steps; s += 2) {   // an odd one's last has zeros
        step(fb, fd);
        step(fd, fb);
    }
    // what is still on its way to LDS ends before the workgroup may
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

    const Place<SA, SB> at_lane = {m0 + wm, n0 + wn, lane};
    if (n0 + BN <= o.N)
        emit<E, true, BA>(o, part, at_lane, acc);
    else
        emit<E, false, BA>(o, part, at_lane, acc);
}

template <typename E, int BM, int BN, int WM, int WN, int STAGES, bool AA, bool BA>
__global__ __launch_bounds__(64 * WM * WN, sizeof(E) == 2 ? 2 : 1) void gemm_fast_kernel(Gemm o) {
    __shared__ __align__(1024) char lds[STAGES][(BM + BN) * kStep * (int)sizeof(E)];
    gemm_fast<E, BM, BN, WM, WN, STAGES, AA, BA>(o, block_of(), lds);
}

// Both of a gradient's products in one launch, where both take the smallest tiles: each
// alone leaves compute units without work at its start and end (1531 x 333 x 1000 in fp32:
// 43 us one after the other, 37 so; all gradients of 1536 x 336 x 1000 46 us, 57 before).
template <typename E, bool FAST>
__global__ __launch_bounds__(kThreads, sizeof(E) == 2 ? 2 : 1) void gemm_pair_kernel(Gemm dx, Gemm dw,
                                                                                   int first) {
    const int at = block_of();
    if constexpr (FAST) {
        __shared__ __align__(1024) char lds[4][128 * kStep * (int)sizeof(E)];
        if (at < first)
            gemm_fast<E, 64, 64, 2, 2, 4, false, true>(dx, at, lds);
        else
            gemm_fast<E, 64, 64, 2, 2, 4, true, true>(dw, at - first, lds);
    } else {
        __shared__ __align__(16) char lds[2 * AnyTile<E, 64, 64>::kBytes];
        if (at < first)
            gemm_any<E, 64, 64, false, true>(dx, at, lds);
        else
            gemm_any<E, 64, 64, true, true>(dw, at - first, lds);
    }
}

// ---- few rows -------------------------------------------------------------------------
// Up to 16 TM rows: what counts is how many of the weights' loads are under way.  A
// workgroup has sixteen columns, a wave an eighth of the sum, whose fragments it loads as
// they are; the eight sums meet in LDS, in order.

constexpr int kFewWaves = 8, kFewAhead = 4;

template <typename E, int TM>
__global__ __launch_bounds__(64 * kFewWaves) void gemm_few_kernel(Gemm o) {
    __shared__ f32x4 part[kFewWaves][TM][64];
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = block_of() * 16;
    if (n0 >= o.N)
        return;
    // steps of 32 positions, as many for each wave as there are; a lane's eight of them lie
    // below K or past it
    const int steps = (o.K + 31) / 32, share = (steps + kFewWaves - 1) / kFewWaves;
    const int first = min(w * share, steps), last = min(first + share, steps);
    const E *b = (const E *)o.b + min(n0 + m, o.N - 1) * o.sb;
    const E *a[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i)
        a[i] = (const E *)o.a + min(16 * i + m, o.M - 1) * o.sa;
    f32x4 acc[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i)
        acc[i] = f32x4{0, 0, 0, 0};
    typedef typename Vec<E, 8>::type Eight;
    for (int s = first; s < last; s += kFewAhead) {
        Frag<E> fb[kFewAhead], fa[kFewAhead][TM];
#pragma unroll
        for (int j = 0; j < kFewAhead; ++j) {
            // past the end, what is there before it, times 0
            const int k = min((s + j) * 32 + 8 * g, o.K - 8);
            fb[j] = *(const Eight *)(b + k);
#pragma unroll
            for (int i = 0; i < TM; ++i)
                fa[j][i] = *(const Eight *)(a[i] + k);
        }
#pragma unroll
        for (int j = 0; j < kFewAhead; ++j) {
            const bool in = s + j < last && (s + j) * 32 + 8 * g < o.K;
            const Frag<E> none = {};
            fb[j] = in ? fb[j] : none;
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                fa[j][i] = in ? fa[j][i] : none;
                acc[i] = mma(fb[j], fa[j][i], acc[i]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i)
        part[w][i][lane] = acc[i];
    __syncthreads();
    if (w >= TM)
        return;
    // a wave a tile of rows
    f32x4 sum = part[0][w][lane];
#pragma unroll
    for (int j = 1; j < kFewWaves; ++j)
        sum += part[j][w][lane];
    const int row = 16 * w + m, col = n0 + 4 * g, count = min(o.N - col, 4);
    if (row >= o.M || count <= 0)
        return;
    float v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r)
        v[r] = sum[r];
    finish<E, 4>(o, row, col, count, v);
    store_upto<E, 4>((E *)o.c + row * o.sc + col, count, v);
}

// The parts of split sums in order, and what follows them.
template <typename E>
__global__ __launch_bounds__(kThreads) void split_sum_kernel(Gemm o, const float *part, E *c,
                                                             int vecs) {
    const long long i = block_of() * (long long)kThreads + threadIdx.x;
    const long long row = i / vecs;
    if (row >= o.M)
        return;
    const int col = (int)(i - row * vecs) * 4, count = min(o.N - col, 4);
    float v[4] = {0, 0, 0, 0};
    for (int p = 0; p < o.split; ++p) {
        float u[4];
        load_upto<float, 4>(part + (p * (long long)o.M + row) * o.N + col, count, u);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            v[r] += u[r];
    }
    finish<E, 4>(o, row, col, count, v);
    store_upto<E, 4>(c + row * o.sc + col, count, v);
}

// ---- d = dy act'(pre), and the sums of its columns -----------------------------------
// d is rounded to the type for the products, whose matrix instructions take no more: in two
// parts both would take twice the time.  The rounding adds to that of dx and dw (2.4e-3 of
// them in the root mean square in bf16, 1.7e-3 where only theirs is).  The sums take it whole.

// Rows of a workgroup, 8 side by side of 32 lanes of 8 columns: as many as leave two
// workgroups a compute unit (gelu' of 1531 x 1000 in fp32: 45 us with 128 rows, 14 with 16).
int sum_rows(int M, int N) {
    int rows = 128;
    while (rows > 16 && cdivll(M, rows) * cdivll(N, 256) < 512)
        rows /= 2;
    return rows;
}

template <typename E>
__global__ __launch_bounds__(kThreads) void act_grad_kernel(const E *dy, long long sdy,
                                                            const E *pre, long long spre, E *d,
                                                            float *sums, int act, int M, int N,
                                                            int slices, int rows) {
    __shared__ float part[8][32 * 8 + 8];
    const int at = block_of(), block = at / slices, slice = at - block * slices;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int col = slice * 256 + lane * 8, count = min(N - col, 8);
    const long long first = (long long)block * rows;
    if (first >= M)
        return;
    float sum[8] = {};
#pragma unroll 4
    for (int i = 0; i < rows / 8; ++i) {
        const long long row = first + i * 8 + w;
        const int have = row < M ? count : 0;
        float v[8];
        load_upto<E, 8>(dy + min(row, (long long)M - 1) * sdy + col, have, v);
        if (act != FINC_ACT_NONE) {
            float p[8];
            load_upto<E, 8>(pre + min(row, (long long)M - 1) * spre + col, have, p);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v[j] *= act_grad(act, p[j]);
            if (have > 0)
                store_upto<E, 8>(d + row * N + col, have, v);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            sum[j] += v[j];
    }
    if (!sums)
        return;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        part[w][lane * 8 + j] = sum[j];
    __syncthreads();
    const int c = slice * 256 + (int)threadIdx.x;
    if (c < N) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            s += part[i][threadIdx.x];
        sums[(long long)block * N + c] = s;
    }
}

// What is left of the gradients, in one launch: the parts of the two products in order, and
// the blocks' sums of the columns of d, in eight shares that are joined in order (as three
// launches 17 us of the gradients of 1531 x 333 x 1000 in fp32, 8 so).
struct Product {
    const float *part;   // (split, M, N)
    void *c;
    long long sc;
    int M, N, split, vecs, blocks;
};
struct Columns {
    const float *sums;   // (rows, N)
    float *out;
    int rows, N, blocks;
};
constexpr int kColumns = 32, kShares = kThreads / kColumns;

template <typename E>
__device__ inline void sum_parts(const Product &p, int block) {
    const long long i = block * (long long)kThreads + threadIdx.x, row = i / p.vecs;
    if (row >= p.M)
        return;
    const int col = (int)(i - row * p.vecs) * 4, count = min(p.N - col, 4);
    float v[4] = {0, 0, 0, 0};
    for (int s = 0; s < p.split; ++s) {
        float u[4];
        load_upto<float, 4>(p.part + (s * (long long)p.M + row) * p.N + col, count, u);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            v[r] += u[r];
    }
    store_upto<E, 4>((E *)p.c + row * p.sc + col, count, v);
}

template <typename E>
__global__ __launch_bounds__(kThreads) void grad_sums_kernel(Product dx, Product dw, Columns db) {
    __shared__ float part[kShares][kColumns];
    int at = block_of();
    if (at < dx.blocks) {
        sum_parts<E>(dx, at);
        return;
    }
    at -= dx.blocks;
    if (at < dw.blocks) {
        sum_parts<E>(dw, at);
        return;
    }
    at -= dw.blocks;
    if (at >= db.blocks)
        return;
    const int lane = threadIdx.x % kColumns, w = threadIdx.x / kColumns, c = at * kColumns + lane;
    const int share = (db.rows + kShares - 1) / kShares;
    const int lo = min(w * share, db.rows), hi = min(lo + share, db.rows);
    float s = 0.0f;
    if (c < db.N) {
#pragma unroll 8
        for (int i = lo; i < hi; ++i)
            s += db.sums[(long long)i * db.N + c];
    }
    part[w][lane] = s;
    __syncthreads();
    if (w == 0 && c < db.N) {
        for (int i = 1; i < kShares; ++i)
            s += part[i][lane];
        db.out[c] = s;
    }
}

// ---- the host --------------------------------------------------------------------------

size_t round256(size_t n) { return (n + 255) / 256 * 256; }
Region rows(const void *p, long long step, long long M, long long D, int size) {
    return {p, M, step, 1, 0, D, size};
}

bool linear_shape(int type, int act, int M, int K, int N) {
    return type_size(type) && act >= FINC_ACT_NONE && act <= FINC_ACT_GELU && M >= 0 && K >= 1 &&
           N >= 1 && M < (1 << 30) && K < (1 << 30) && N < (1 << 30) &&
           (long long)M * N < (1ll << 40) && (long long)M * K < (1ll << 40) &&
           (long long)K * N < (1ll << 40);
}

// Rows of n elements that are whole chunks of 16 bytes, and whether they also start at
// multiples of 16 bytes.
bool chunks(int n, int size) { return (long long)n * size % 16 == 0; }
bool aligned(const void *p, long long s, int size) {
    return (uintptr_t)p % 16 == 0 && s * size % 16 == 0;
}

// Square tiles of the kernels, and microseconds that 32 positions of the sum take: of a
// tile alone on a compute unit (along the sum, and with an operand across it, whose rows
// come from more places), and of each of `side` tiles side by side there.
struct Tile {
    int dim, side;
    double alone, across, each;
};
// 16 bits: 2048 x 1024 x 1024 forward takes 11 us with tiles of 64 and 14 with 128; 4096 x
// 2048 x 2048 takes 75, 42 and 50 with 64, 128 and 256; 32768 x 1024 x 4096 257 with 256.
const Tile kFast16[] = {{64, 4, 0.13, 0.45, 0.13}, {128, 2, 0.30, 0.58, 0.30},
                        {256, 1, 0.87, 0.97, 0.87}};
// 32: 8192 x 2048 x 2048 632 with 64, 557 with 128; 1536 x 336 x 1000 19 and 31.
const Tile kFast32[] = {{64, 4, 0.65, 0.65, 0.58}, {128, 1, 2.2, 2.2, 2.2}};
// Operands of any alignment: 8191 x 1001 x 1003 58 and 46 in 16 bits, 177 and 159 in 32.
const Tile kAny16[] = {{64, 4, 0.55, 0.55, 0.22}, {128, 2, 1.1, 1.1, 0.68}};
const Tile kAny32[] = {{64, 4, 1.55, 1.55, 0.69}, {128, 2, 4.0, 4.0, 2.4}};

// Tile and split of a product: the cheapest of all by that and by what a launch, a tile's
// end and the parts of split sums cost (6 us and their way to memory and back at 4 TB/s: 64
// rows by 2048 x 2048 in bf16 take 9.2 us in four parts in a graph and 11.6 in one, but a
// call outside one 14.4, for its second launch, and 11.9).  The gradient of
// 2048 x 2048 weights over 16384 rows, alone and with the joining of its parts: 150 us in four
// parts with tiles of 256, 167 in two with 128, 242 in one with 64; of 64 x 256 over 32768: 456
// in one part, 38 in sixteen.
struct Plan {
    int dim, split, per;
    bool fast;
};
// of parts of `per` positions of the sum
double cost(const Tile &t, int M, int N, int parts, int per, bool across) {
    const double tiles = (double)cdivll(M, t.dim) * cdivll(N, t.dim);
    const double n = ceil(tiles * parts / 256.0), side = n < t.side ? n : t.side;
    const double step = (across ? t.across : t.alone) > side * t.each ? (across ? t.across : t.alone)
                                                                      : side * t.each;
    const double us = ceil(n / t.side) * (per / 32.0) * step + n * t.dim * t.dim / 16384.0;
    return parts > 1 ? us + (6.0 + parts * (double)M * N * 8.0 / 4e6) : us;
}
// The parts, which set the sums' order, follow from type and sizes alone: operands whose rows
// are whole chunks have the same ones at every address, also where they go by the kernel of any
// alignment, whose best ones are others (64 rows by 2048 x 2048 in bf16 an element behind such an
// address: 23 us, 14 with parts of its own; 256 by 4096 x 4096 53 and 33; most sizes the same).
Plan plan(int M, int N, int K, int size, bool whole, bool across, bool fast) {
    const Tile *from = whole ? (size == 2 ? kFast16 : kFast32) : (size == 2 ? kAny16 : kAny32);
    const int kinds = whole && size == 2 ? 3 : 2, sum = K > 0 ? K : 1;   // none: zeros
    Plan best = {};
    double least = 0.0;
    for (int k = 0; k < kinds; ++k)
        for (int split = 1; split <= 64; split *= 2) {
            if (split > 1 && sum / split < 128)
                break;
            const int per = (int)(cdivll(cdivll(sum, split), 64) * 64);
            const int parts = (int)cdivll(sum, per);
            const double us = cost(from[k], M, N, parts, per, across);
            if (best.dim == 0 || us < least) {
                least = us;
                best.dim = from[k].dim;
                best.split = parts;
                best.per = per;
            }
        }
    best.fast = whole && fast;
    if (whole && !fast) {
        const Tile *any = size == 2 ? kAny16 : kAny32;
        best.dim = cost(any[0], M, N, best.split, best.per, across) <=
                           cost(any[1], M, N, best.split, best.per, across)
                       ? any[0].dim
                       : any[1].dim;
    }
    return best;
}
// whole: both operands' rows are whole chunks.
size_t split_bytes(int M, int N, int K, int size, bool whole, bool across) {
    const int split = plan(M, N, K, size, whole, across, true).split;
    return split > 1 ? round256((size_t)split * M * N * 4) : 0;
}

template <typename E, bool AA, bool BA>
void launch_gemm(const Plan &p, const Gemm &o, dim3 grid, hipStream_t stream) {
    if constexpr (sizeof(E) == 2)
        if (p.fast && p.dim == 256) {
            gemm_fast_kernel<E, 256, 256, 2, 4, 4, AA, BA><<<grid, 512, 0, stream>>>(o);
            return;
        }
    if (p.fast && p.dim == 128)
        gemm_fast_kernel<E, 128, 128, 2, 2, 4, AA, BA><<<grid, 256, 0, stream>>>(o);
    else if (p.fast)
        // more stages hide more of a short row of tiles' latency (256 x 4096 x 4096 bf16 21
        // us, 28 with four), but take the places of tiles side by side
        gemm_fast_kernel<E, 64, 64, 2, 2, sizeof(E) == 2 && !BA ? 6 : 4, AA, BA>
            <<<grid, 256, 0, stream>>>(o);
    else if (p.dim == 128)
        gemm_kernel<E, 128, 128, AA, BA><<<grid, kThreads, 0, stream>>>(o);
    else
        gemm_kernel<E, 64, 64, AA, BA><<<grid, kThreads, 0, stream>>>(o);
}

// Whether the kernel of few rows is the faster one (2048 x 2048 in bf16: 4.6 us for one row,
// 6.0 for sixteen and 7.9 for 32, by tiles 7.7, 8.9 and 9.3; 2048 x 16384: 13.9, 17.9 and
// 24.9 against 15.8, 16.3 and 16.5; sums over 8192: 10.8 and 16.3 against 10.7 and 12.6).
bool few(int M, int N, int K) {
    return K % 8 == 0 && K <= 4096 &&   // a lane's eight positions at once
           (M == 1 || (M <= 32 && cdivll(M, 16) * N * (long long)K <= 1ll << 24));
}

// Sets the product's tiles and parts.
template <bool AA, bool BA>
Plan planned(int type, Gemm &o) {
    const int sz = type_size(type);
    const Plan p = plan(o.M, o.N, o.K, sz,
                        chunks(AA ? o.M : o.K, sz) && chunks(BA ? o.N : o.K, sz), BA,
                        aligned(o.a, o.sa, sz) && aligned(o.b, o.sb, sz));
    o.split = p.split;
    o.per = p.per;
    o.tiles_m = (int)cdivll(o.M, p.dim);
    o.tiles_n = (int)cdivll(o.N, p.dim);
    return p;
}
long long groups_of(const Gemm &o) { return (long long)o.tiles_m * o.tiles_n * o.split; }
Gemm into(Gemm o, void *c) {
    o.c = c;
    return o;
}

// The product, or its parts in `workspace`.
template <bool AA, bool BA>
void run_gemm(int type, const Plan &p, const Gemm &o, void *workspace, hipStream_t stream) {
    const Gemm part = into(o, o.split > 1 ? workspace : o.c);
    with_type(type, [&](auto e) {
        launch_gemm<decltype(e), AA, BA>(p, part, grid_of(groups_of(o)), stream);
    });
}
long long sum_groups(int M, int vecs) { return cdivll((long long)M * vecs, kThreads); }

int sum_blocks(int M, int N) { return (int)cdivll(M, sum_rows(M, N)); }

}  // namespace

extern "C" {

size_t finc_linear_workspace_bytes(int type, int M, int K, int N) {
    const int sz = type_size(type);
    return linear_shape(type, FINC_ACT_NONE, M, K, N) ? split_bytes(M, N, K, sz, chunks(K, sz), false)
                                                       : 0;
}

int finc_linear_forward(const finc_linear_args *a, hipStream_t stream) {
    if (!a || !linear_shape(a->type, a->act, a->M, a->K, a->N) || ((uintptr_t)a->workspace & 255u))
        return FINC_EINVAL;
    const int sz = type_size(a->type), M = a->M, K = a->K, N = a->N;
    const bool same = a->residual && a->residual == a->y;
    if (same && M > 1 && a->sres != a->sy)
        return FINC_EINVAL;
    const Region in[] = {rows(a->x, a->sx, M, K, sz), rows(a->w, a->sw, N, K, sz),
                         flat(a->bias, a->bias ? N : 0, 4),
                         rows(same ? nullptr : a->residual, a->sres, a->residual && !same ? M : 0,
                              N, sz)};
    const Region out[] = {rows(a->y, a->sy, M, N, sz), rows(a->pre, a->spre, a->pre ? M : 0, N, sz),
                          flat(a->workspace,
                               (long long)finc_linear_workspace_bytes(a->type, M, K, N), 1)};
    for (const Region &r : in)
        if (!readable(r))
            return FINC_EINVAL;
    for (const Region &r : out)
        if (!writable(r))
            return FINC_EINVAL;
    if (!disjoint(in, out))
        return FINC_EINVAL;
    if (M == 0)
        return FINC_OK;
    Gemm o = {};
    o.a = a->x;
    o.sa = a->sx;
    o.b = a->w;
    o.sb = a->sw;
    o.c = a->y;
    o.sc = a->sy;
    o.bias = a->bias;
    o.residual = a->residual;
    o.sr = a->sres;
    o.pre = a->pre;
    o.sp = a->spre;
    o.M = M;
    o.N = N;
    o.K = K;
    o.act = a->act;
    const Plan p = planned<false, false>(a->type, o);
    if (few(M, N, K)) {
        o.split = 1;
        with_type(a->type, [&](auto e) {
            typedef decltype(e) E;
            const dim3 grid = grid_of(cdivll(N, 16));
            if (M <= 16)
                gemm_few_kernel<E, 1><<<grid, 64 * kFewWaves, 0, stream>>>(o);
            else
                gemm_few_kernel<E, 2><<<grid, 64 * kFewWaves, 0, stream>>>(o);
        });
        return launched();
    }
    run_gemm<false, false>(a->type, p, o, a->workspace, stream);
    if (o.split > 1)
        with_type(a->type, [&](auto e) {
            typedef decltype(e) E;
            const int vecs = (N + 3) / 4;
            split_sum_kernel<E><<<grid_of(sum_groups(M, vecs)), kThreads, 0, stream>>>(
                o, (const float *)a->workspace, (E *)o.c, vecs);
        });
    return launched();
}

size_t finc_linear_grad_workspace_bytes(int type, int act, int M, int K, int N) {
    if (!linear_shape(type, act, M, K, N))
        return 0;
    const int sz = type_size(type);
    const bool whole = chunks(N, sz) && chunks(K, sz);
    const size_t x = split_bytes(M, K, N, sz, whole, true), w = split_bytes(N, K, M, sz, whole, true);
    return (act != FINC_ACT_NONE ? round256((size_t)M * N * sz) : 0) +
           round256((size_t)sum_blocks(M, N) * N * 4) + x + w;
}

int finc_linear_backward(const finc_linear_grad_args *a, hipStream_t stream) {
    if (!a || !linear_shape(a->type, a->act, a->M, a->K, a->N) || ((uintptr_t)a->workspace & 255u))
        return FINC_EINVAL;
    const int sz = type_size(a->type), M = a->M, K = a->K, N = a->N;
    const bool act = a->act != FINC_ACT_NONE;
    const Region in[] = {rows(a->dy, a->sdy, M, N, sz), rows(a->x, a->sx, a->dw ? M : 0, K, sz),
                         rows(a->w, a->sw, a->dx ? N : 0, K, sz),
                         rows(a->pre, a->spre, act ? M : 0, N, sz)};
    const Region out[] = {
        rows(a->dx, a->sdx, a->dx ? M : 0, K, sz), rows(a->dw, a->sdw, a->dw ? N : 0, K, sz),
        flat(a->dbias, a->dbias ? N : 0, 4),
        flat(a->workspace, (long long)finc_linear_grad_workspace_bytes(a->type, a->act, M, K, N), 1)};
    for (const Region &r : in)
        if (!readable(r))
            return FINC_EINVAL;
    for (const Region &r : out)
        if (!writable(r))
            return FINC_EINVAL;
    if (!disjoint(in, out))
        return FINC_EINVAL;
    char *ws = (char *)a->workspace;
    auto take = [&](size_t bytes) {
        char *p = ws;
        ws += round256(bytes);
        return p;
    };
    void *d = act ? take((size_t)M * N * sz) : nullptr;
    const int blocks = sum_blocks(M, N), slices = (N + 255) / 256;
    float *sums = (float *)take((size_t)blocks * N * 4);
    // one block's sums are the columns'
    Columns db = {sums, a->dbias, blocks, N, 0};
    if (a->dbias && blocks != 1)
        db.blocks = (int)cdivll(N, kColumns);
    if (M > 0 && (act || a->dbias))
        with_type(a->type, [&](auto e) {
            typedef decltype(e) E;
            act_grad_kernel<E><<<grid_of((long long)blocks * slices), kThreads, 0, stream>>>(
                (const E *)a->dy, a->sdy, (const E *)a->pre, a->spre, (E *)d,
                a->dbias && blocks == 1 ? a->dbias : (a->dbias ? sums : nullptr), a->act, M, N,
                slices, sum_rows(M, N));
        });
    Product dx = {}, dw = {};
    auto parts = [&](const Gemm &o) {
        Product p = {};
        if (o.split > 1) {
            const int vecs = (o.N + 3) / 4;
            p = {(const float *)ws, o.c, o.sc, o.M, o.N, o.split, vecs,
                 (int)sum_groups(o.M, vecs)};
            take((size_t)o.split * o.M * o.N * 4);
        }
        return p;
    };
    Gemm x = {}, w = {};
    Plan px = {}, pw = {};
    x.a = w.a = act ? d : a->dy;
    x.sa = w.sa = act ? N : a->sdy;
    const bool any_x = a->dx && M > 0;
    if (any_x) {
        x.b = a->w;
        x.sb = a->sw;
        x.c = a->dx;
        x.sc = a->sdx;
        x.M = M;
        x.N = K;
        x.K = N;
        px = planned<false, true>(a->type, x);
        dx = parts(x);
    }
    if (a->dw) {
        w.b = a->x;
        w.sb = a->sx;
        w.c = a->dw;
        w.sc = a->sdw;
        w.M = N;
        w.N = K;
        w.K = M;
        pw = planned<true, true>(a->type, w);
        dw = parts(w);
    }
    if (any_x && a->dw && px.dim == 64 && pw.dim == 64 && px.fast == pw.fast)
        with_type(a->type, [&](auto e) {
            typedef decltype(e) E;
            const Gemm ox = into(x, dx.blocks ? (void *)dx.part : x.c),
                       ow = into(w, dw.blocks ? (void *)dw.part : w.c);
            const dim3 grid = grid_of(groups_of(x) + groups_of(w));
            if (px.fast)
                gemm_pair_kernel<E, true><<<grid, kThreads, 0, stream>>>(ox, ow, (int)groups_of(x));
            else
                gemm_pair_kernel<E, false><<<grid, kThreads, 0, stream>>>(ox, ow, (int)groups_of(x));
        });
    else {
        if (any_x)
            run_gemm<false, true>(a->type, px, x, (void *)dx.part, stream);
        if (a->dw)
            run_gemm<true, true>(a->type, pw, w, (void *)dw.part, stream);
    }
    const long long groups = (long long)dx.blocks + dw.blocks + db.blocks;
    if (groups > 0)
        with_type(a->type, [&](auto e) {
            grad_sums_kernel<decltype(e)><<<grid_of(groups), kThreads, 0, stream>>>(dx, dw, db);
        });
    return launched();
}

}  // extern "C"
