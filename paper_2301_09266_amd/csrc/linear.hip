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

// The normal distribution's function: half of erfc on both sides, so that far negative p
// keep its relative precision.
__device__ inline float normal_cdf(float p) { return 0.5f * erfcf(-0.70710678118654752f * p); }
__device__ inline float act_value(int act, float p) {
    switch (act) {
    case FINC_ACT_RELU:
        return p < 0.0f ? 0.0f : p;   // NaN stays
    case FINC_ACT_SILU:
        return silu(p);
    case FINC_ACT_GELU:
        return __builtin_fmaxf(p, -1e30f) * normal_cdf(p);
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
        const float q = __builtin_amdgcn_fmed3f(p, -1e15f, 1e15f);
        return normal_cdf(p) + q * 0.39894228040143268f * exp_fast(-0.5f * q * q);
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
template <typename E, int BM, int BN, bool AA, bool BA>
__global__ __launch_bounds__(kThreads) void gemm_kernel(Gemm o) {
    constexpr int BK = 128 / sizeof(E), TM = BM / 32, TN = BN / 32;
    typedef Operand<E, BM, BK, AA> OA;
    typedef Operand<E, BN, BK, BA> OB;
    __shared__ __align__(16) E sa[OA::kOuter * OA::kLd];
    __shared__ __align__(16) E sb[OB::kOuter * OB::kLd];
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int at = block_of();
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
            if (o.bias) {
                float u[4];
                load_upto<float, 4>(o.bias + col, count, u);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    v[r] += u[r];
            }
            if (o.pre)
                store_upto<E, 4>((E *)o.pre + row * o.sp + col, count, v);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                v[r] = act_value(o.act, v[r]);
            if (o.residual) {
                float u[4];
                load_upto<E, 4>((const E *)o.residual + row * o.sr + col, count, u);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    v[r] += u[r];
            }
            store_upto<E, 4>((E *)o.c + row * o.sc + col, count, v);
        }
    }
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
    if (o.bias) {
        float u[4];
        load_upto<float, 4>(o.bias + col, count, u);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            v[r] += u[r];
    }
    if (o.pre)
        store_upto<E, 4>((E *)o.pre + row * o.sp + col, count, v);
#pragma unroll
    for (int r = 0; r < 4; ++r)
        v[r] = act_value(o.act, v[r]);
    if (o.residual) {
        float u[4];
        load_upto<E, 4>((const E *)o.residual + row * o.sr + col, count, u);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            v[r] += u[r];
    }
    store_upto<E, 4>(c + row * o.sc + col, count, v);
}

// ---- d = dy act'(pre), and the sums of its columns -----------------------------------

constexpr int kSumRows = 128;   // rows of a workgroup: 8 side by side of 32 lanes of 8 columns

template <typename E>
__global__ __launch_bounds__(kThreads) void act_grad_kernel(const E *dy, long long sdy,
                                                            const E *pre, long long spre, E *d,
                                                            float *sums, int act, int M, int N,
                                                            int slices) {
    __shared__ float part[8][32 * 8 + 8];
    const int at = block_of(), block = at / slices, slice = at - block * slices;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int col = slice * 256 + lane * 8, count = min(N - col, 8);
    const long long first = (long long)block * kSumRows;
    if (first >= M)
        return;
    float sum[8] = {};
#pragma unroll 4
    for (int i = 0; i < kSumRows / 8; ++i) {
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

// The blocks' sums in order: 4 shares a column, joined in order.
__global__ __launch_bounds__(kThreads) void column_sum_kernel(const float *sums, float *out, int N,
                                                              int blocks) {
    __shared__ float part[4][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    const int share = (blocks + 3) / 4, lo = min(w * share, blocks), hi = min(lo + share, blocks);
    float s = 0.0f;
    if (c < N)
        for (int i = lo; i < hi; ++i)
            s += sums[(long long)i * N + c];
    part[w][lane] = s;
    __syncthreads();
    if (w == 0 && c < N)
        out[c] = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
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

// Tile and split of a product.
struct Plan {
    int tile, split, per;
};
Plan plan(int M, int N, int K) {
    Plan p;
    p.tile = cdivll(M, 128) * cdivll(N, 128) >= 256 ? 128 : 64;
    const long long tiles = cdivll(M, p.tile) * cdivll(N, p.tile);
    p.split = 1;
    while (p.split < 16 && tiles * p.split < 256 && K / (p.split * 2) >= 256)
        p.split *= 2;
    p.per = (int)(cdivll(cdivll(K > 0 ? K : 1, p.split), 64) * 64);
    p.split = (int)cdivll(K > 0 ? K : 1, p.per);   // an empty sum is one of zeros
    return p;
}
size_t split_bytes(int M, int N, int K) {
    const Plan p = plan(M, N, K);
    return p.split > 1 ? round256((size_t)p.split * M * N * 4) : 0;
}

template <bool AA, bool BA>
void run_gemm(int type, Gemm o, void *workspace, hipStream_t stream) {
    const Plan p = plan(o.M, o.N, o.K);
    o.split = p.split;
    o.per = p.per;
    o.tiles_m = (int)cdivll(o.M, p.tile);
    o.tiles_n = (int)cdivll(o.N, p.tile);
    void *c = o.c;
    if (p.split > 1)
        o.c = workspace;
    const dim3 grid = grid_of((long long)o.tiles_m * o.tiles_n * p.split);
    with_type(type, [&](auto e) {
        typedef decltype(e) E;
        if (p.tile == 128)
            gemm_kernel<E, 128, 128, AA, BA><<<grid, kThreads, 0, stream>>>(o);
        else
            gemm_kernel<E, 64, 64, AA, BA><<<grid, kThreads, 0, stream>>>(o);
        if (p.split > 1) {
            const int vecs = (o.N + 3) / 4;
            split_sum_kernel<E><<<grid_of(cdivll((long long)o.M * vecs, kThreads)), kThreads, 0,
                                  stream>>>(o, (const float *)workspace, (E *)c, vecs);
        }
    });
}

int sum_blocks(int M) { return (int)cdivll(M, kSumRows); }

}  // namespace

extern "C" {

size_t finc_linear_workspace_bytes(int type, int M, int K, int N) {
    return linear_shape(type, FINC_ACT_NONE, M, K, N) ? split_bytes(M, N, K) : 0;
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
    run_gemm<false, false>(a->type, o, a->workspace, stream);
    return launched();
}

size_t finc_linear_grad_workspace_bytes(int type, int act, int M, int K, int N) {
    if (!linear_shape(type, act, M, K, N))
        return 0;
    const size_t x = split_bytes(M, K, N), w = split_bytes(N, K, M);
    return (act != FINC_ACT_NONE ? round256((size_t)M * N * type_size(type)) : 0) +
           round256((size_t)sum_blocks(M) * N * 4) + (x > w ? x : w);
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
    float *sums = (float *)take((size_t)sum_blocks(M) * N * 4);
    const int blocks = sum_blocks(M), slices = (N + 255) / 256;
    if (M > 0 && (act || a->dbias))
        with_type(a->type, [&](auto e) {
            typedef decltype(e) E;
            act_grad_kernel<E><<<grid_of((long long)blocks * slices), kThreads, 0, stream>>>(
                (const E *)a->dy, a->sdy, (const E *)a->pre, a->spre, (E *)d,
                a->dbias ? sums : nullptr, a->act, M, N, slices);
        });
    if (a->dbias)
        column_sum_kernel<<<(N + 63) / 64, kThreads, 0, stream>>>(sums, a->dbias, N, blocks);
    Gemm o = {};
    o.a = act ? d : a->dy;
    o.sa = act ? N : a->sdy;
    if (a->dx && M > 0) {
        o.b = a->w;
        o.sb = a->sw;
        o.c = a->dx;
        o.sc = a->sdx;
        o.M = M;
        o.N = K;
        o.K = N;
        run_gemm<false, true>(a->type, o, ws, stream);
    }
    if (a->dw) {
        o.b = a->x;
        o.sb = a->sx;
        o.c = a->dw;
        o.sc = a->sdw;
        o.M = N;
        o.N = K;
        o.K = M;
        run_gemm<true, true>(a->type, o, ws, stream);
    }
    return launched();
}

}  // extern "C"
