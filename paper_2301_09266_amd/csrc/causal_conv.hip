// causal_conv.hip -- the short causal convolution along every channel's raster,
// its gradients and its single-position form (finc_causal_conv_* of finc.h).
//
// y[t] = act(bias + sum_j w[j] e[t + j]) with e the K - 1 inputs before the
// raster followed by the raster: every value is read once and written once, so
// the kernels are bound by memory.  A thread takes 16 bytes of one row and the
// H >= K - 1 elements before them (which a neighbour has in flight: they come
// from L1), so no value goes through LDS and a tile has no halo to wait for.
// The gradients take the same tile with H elements on both sides: the K - 1
// gradients of the pre-activation to the right of the tile are recomputed.
#include "seq_common.h"

namespace {

using namespace finc_seq;

constexpr int kThreads = 256;

// Elements before a tile: a power of two, so that they load as one vector.
template <int K>
constexpr int kHalo = K <= 1 ? 1 : K <= 2 ? 1 : K <= 3 ? 2 : K <= 5 ? 4 : 8;

// Elements a thread takes: 16 bytes forward; twice that for the gradients, which
// recompute K - 1 gradients beside them (8 x 2048 x 4096 in bf16, K 4: 113 us, and 132
// with 16 bytes; 300 x 9000, where few threads are left, 11.2 and 9.4; with the loads
// together 97 and 10.8).
constexpr int kTileBytes(bool back) { return back ? 32 : 16; }
template <typename E, bool BACK>
constexpr int kTile = kTileBytes(BACK) / (int)sizeof(E);

struct ConvArgs {
    const void *x, *dy, *state, *dstate_out;
    void *y, *dx, *state_out, *dstate;
    const float *w, *bias;
    float *partial;          // the parts' sums, K + 1 for every channel
    const int *lengths;
    long long xb, xd, yb, yd, gb, gd, ob, od;
    int B, D, L;
    int txl, tiles_t, tiles_r;   // threads along the row (log2), tiles of t and of rows
    int parts;
    FastDiv div_d, div_t;
};

__device__ inline int row_length(const int *lengths, int b, int L) {
    return lengths ? min(max(lengths[b], 0), L) : L;
}

// N elements as they lie in memory, 0 in lanes where `ok` is false.  The loads of a tile
// are all under way before the first is converted.
template <typename E, int N>
__device__ inline typename Vec<E, N>::type load_raw(const E *p, bool ok) {
    typename Vec<E, N>::type v = {};
    if (ok)
        v = *(const typename Vec<E, N>::type *)p;
    return v;
}
template <typename E, int N>
__device__ inline void convert(typename Vec<E, N>::type t, float *v) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        v[i] = (float)t[i];
}

// The H elements before t0 < H: of x, of the state (K - 1 elements) or 0.
template <typename E, int K, int H>
__device__ inline void load_first(const E *x, const E *state, int t0, float *v) {
#pragma unroll
    for (int i = 0; i < H; ++i) {
        const int t = t0 - H + i;
        v[i] = t >= 0 ? (float)x[t] : state && t >= 1 - K ? (float)state[K - 1 + t] : 0.0f;
    }
}

// One tile a thread, rows side by side in a workgroup where they are short.  64 x 512
// rows of 256 in fp32, K 4: 17 us, 3.9 TB/s of the 4.8 that a copy reaches.
template <typename E, int K, bool SILU>
__global__ __launch_bounds__(kThreads) void conv_forward_kernel(ConvArgs a) {
    constexpr int V = kTile<E, false>, H = kHalo<K>;
    const int tx = 1 << a.txl;
    const int blk = block_of(), rt = fdiv(blk, a.div_t), tt = blk - rt * a.tiles_t;
    const long long row = (long long)rt * (kThreads >> a.txl) + (threadIdx.x >> a.txl);
    if (row >= (long long)a.B * a.D)
        return;
    const int b = fdiv((int)row, a.div_d), d = (int)row - b * a.D;
    const long long t0l = ((long long)tt * tx + (threadIdx.x & (tx - 1))) * V;
    const E *x = (const E *)a.x + (b * a.xb + d * a.xd);
    const E *state = a.state ? (const E *)a.state + row * (K - 1) : nullptr;
    const int n = row_length(a.lengths, b, a.L);
    if (t0l >= a.L && t0l > 0)
        return;
    const int t0 = (int)t0l;
    float v[H + V], y[V];
    const bool whole = t0 + V <= a.L;
    const auto before = load_raw<E, H>(x + (t0 - H), t0 >= H);
    const auto tile = load_raw<E, V>(x + t0, whole);
    const float bias = a.bias ? a.bias[d] : 0.0f;
    float w[K];
#pragma unroll
    for (int j = 0; j < K; ++j)
        w[j] = a.w[(long long)d * K + j];
    convert<E, H>(before, v);
    convert<E, V>(tile, v + H);
    if (t0 < H)
        load_first<E, K, H>(x, state, t0, v);
    if (!whole)
        load_upto<E, V>(x + t0, a.L - t0, v + H);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float p = bias;
#pragma unroll
        for (int j = 0; j < K; ++j)
            p = __builtin_fmaf(w[j], v[H - (K - 1) + i + j], p);
        y[i] = keep_if(t0 + i < n, SILU ? silu(p) : p);
    }
    store_upto<E, V>((E *)a.y + (b * a.yb + d * a.yd) + t0, a.L - t0, y);
    if (t0 == 0 && a.state_out) {
        E *out = (E *)a.state_out + row * (K - 1);
#pragma unroll
        for (int e = 0; e < K - 1; ++e) {
            const int t = n - (K - 1) + e;
            out[e] = t >= 0 ? x[t] : state ? state[K - 1 + t] : (E)0.0f;
        }
    }
}

// One channel and a part of its (row, tile) pairs: dx of the part, and the part's
// sums for dw and dbias, which stay in registers until the part ends.  Bound by memory:
// 8 x 2048 x 4096 in bf16, K 4, in 97 us in a graph and 88 call by call, 4.2 and 4.6 TB/s
// (111 in a graph with each load waited for by itself).
template <typename E, int K, bool SILU>
__global__ __launch_bounds__(kThreads) void conv_backward_kernel(ConvArgs a) {
    constexpr int V = kTile<E, true>, H = kHalo<K>, Q = K - 1;
    __shared__ float red[K + 1][kThreads / 64];
    const int tx = 1 << a.txl, ty = kThreads >> a.txl;
    const int blk = block_of(), part = fdiv(blk, a.div_d), d = blk - part * a.D;
    const int lx = threadIdx.x & (tx - 1), ly = threadIdx.x >> a.txl;
    if (part >= a.parts)
        return;
    float w[K], dw[K], db = 0.0f;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        w[j] = a.w[(long long)d * K + j];
        dw[j] = 0.0f;
    }
    const float bias = a.bias ? a.bias[d] : 0.0f;
    for (int u = part; u < a.tiles_r * a.tiles_t; u += a.parts) {
        const int rt = fdiv(u, a.div_t), tt = u - rt * a.tiles_t;
        const int b = rt * ty + ly;
        const long long t0l = ((long long)tt * tx + lx) * V;
        // a thread without a row or a tile has nothing to add
        if (b >= a.B || (t0l >= a.L && t0l > 0))
            continue;
        const int t0 = (int)t0l;
        const int n = row_length(a.lengths, b, a.L);
        const E *x = (const E *)a.x + (b * a.xb + d * a.xd);
        const E *dy = (const E *)a.dy + (b * a.gb + d * a.gd);
        const long long row = (long long)b * a.D + d;
        const E *state = a.state ? (const E *)a.state + row * Q : nullptr;
        const E *dso = a.dstate_out ? (const E *)a.dstate_out + row * Q : nullptr;
        float v[H + V + H], g[V + H];
        {
            const bool whole = t0 + V <= a.L, more = t0 + V + H <= a.L;
            const auto before = load_raw<E, H>(x + (t0 - H), t0 >= H);
            const auto xt = load_raw<E, V>(x + t0, whole), gt = load_raw<E, V>(dy + t0, whole);
            const auto xa = load_raw<E, H>(x + t0 + V, more), ga = load_raw<E, H>(dy + t0 + V, more);
            convert<E, H>(before, v);
            convert<E, V>(xt, v + H);
            convert<E, H>(xa, v + H + V);
            convert<E, V>(gt, g);
            convert<E, H>(ga, g + V);
            if (t0 < H)
                load_first<E, K, H>(x, state, t0, v);
            if (!whole) {
                load_upto<E, V>(x + t0, a.L - t0, v + H);
                load_upto<E, V>(dy + t0, a.L - t0, g);
            } else if (!more && t0 + V < a.L) {
                load_upto<E, H>(x + t0 + V, a.L - t0 - V, v + H + V);
                load_upto<E, H>(dy + t0 + V, a.L - t0 - V, g + V);
            }
        }
        if (SILU) {
#pragma unroll
            for (int i = 0; i < V + Q; ++i) {
                float p = bias;
#pragma unroll
                for (int j = 0; j < K; ++j)
                    p = __builtin_fmaf(w[j], v[H - Q + i + j], p);
                g[i] *= silu_grad(p, sigmoid(p));
            }
        }
        if (t0 + V + H > n) {   // padding may hold anything
#pragma unroll
            for (int i = 0; i < V + H; ++i)
                g[i] = keep_if(t0 + i < n, g[i]);
        }
        float dx[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float s = 0.0f;
#pragma unroll
            for (int j = 0; j < K; ++j)
                s = __builtin_fmaf(w[j], g[i + Q - j], s);
            dx[i] = s;
        }
        // Padding adds nothing, not even 0 times the inputs before it, which may be infinite
        // or NaN: an empty row's state, the row's last inputs, padding itself.
        if (t0 + V <= n) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                db += g[i];
#pragma unroll
                for (int j = 0; j < K; ++j)
                    dw[j] = __builtin_fmaf(g[i], v[H - Q + i + j], dw[j]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                db += g[i];
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    const float s = __builtin_fmaf(g[i], v[H - Q + i + j], dw[j]);
                    dw[j] = t0 + i < n ? s : dw[j];
                }
            }
        }
        if (t0 + V + Q > n) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int t = t0 + i;
                if (dso && t < n && t + Q >= n)
                    dx[i] += (float)dso[t + Q - n];
                dx[i] = keep_if(t < n, dx[i]);
            }
        }
        store_upto<E, V>((E *)a.dx + (b * a.ob + d * a.od) + t0, a.L - t0, dx);
        if (t0 == 0 && a.dstate) {
            E *ds = (E *)a.dstate + row * Q;
#pragma unroll
            for (int e = 0; e < Q; ++e) {
                float s = dso && e >= n ? (float)dso[e - n] : 0.0f;
#pragma unroll
                for (int t = 0; t <= e; ++t)
                    s = __builtin_fmaf(w[e - t], g[t], s);
                ds[e] = (E)s;
            }
        }
    }
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j <= K; ++j) {
        const float s = wave_sum(j < K ? dw[j < K ? j : 0] : db);
        if ((threadIdx.x & 63) == 0)
            red[j][wave] = s;
    }
    __syncthreads();
    if (threadIdx.x <= K) {
        const float *r = red[threadIdx.x];
        a.partial[((long long)part * a.D + d) * (K + 1) + threadIdx.x] =
            (r[0] + r[1]) + (r[2] + r[3]);
    }
}

// dw and dbias: the parts' sums, eight groups of parts in turn, then the groups in
// order (5 us, its launch and latencies, for 2048 channels).
__global__ __launch_bounds__(256) void conv_sum_kernel(const float *partial, int parts, float *dw,
                                                       float *dbias, int D, int K) {
    __shared__ float red[8][33];
    const long long n = (long long)D * (K + 1);
    const int l = threadIdx.x & 31, grp = threadIdx.x >> 5;
    const long long e = block_of() * 32ll + l;
    float s = 0.0f;
    if (e < n)
        for (int p = grp; p < parts; p += 64) {
            float v[8];   // in flight together
#pragma unroll
            for (int k = 0; k < 8; ++k)
                v[k] = partial[min(p + 8 * k, parts - 1) * n + e];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                s += p + 8 * k < parts ? v[k] : 0.0f;
        }
    red[grp][l] = s;
    __syncthreads();
    if (grp == 0 && e < n) {
        s = 0.0f;
        for (int i = 0; i < 8; ++i)
            s += red[i][l];
        const int d = (int)(e / (K + 1)), j = (int)(e - (long long)d * (K + 1));
        if (j < K)
            dw[(long long)d * K + j] = s;
        else if (dbias)
            dbias[d] = s;
    }
}

// One position: a thread a (row, channel), whose K - 1 earlier inputs move up by one in
// place.  64 x 2048 in bf16: 4 us in a graph, a launch and the way to the slot and its state.
template <typename E>
__global__ __launch_bounds__(kThreads) void conv_step_kernel(const E *x, long long sx, E *y,
                                                             long long sy, const float *w,
                                                             const float *bias, E *state,
                                                             const int *slots, int B, int S, int D,
                                                             int K, int silu_on) {
    const int d = blockIdx.x * kThreads + threadIdx.x;
    if (d >= D)
        return;
    for (int b = blockIdx.y; b < B; b += gridDim.y) {
        const int slot = slots ? slots[b] : b;
        E *out = y + (long long)b * sy + d;
        if (slot < 0 || slot >= S) {
            *out = (E)0.0f;
            continue;
        }
        E *st = state + ((long long)slot * D + d) * (K - 1);
        const E in = x[(long long)b * sx + d];
        E old[FINC_MAX_TAPS - 1];
#pragma unroll
        for (int j = 0; j < FINC_MAX_TAPS - 1; ++j)
            if (j < K - 1)
                old[j] = st[j];
        float p = bias ? bias[d] : 0.0f;
#pragma unroll
        for (int j = 0; j < FINC_MAX_TAPS - 1; ++j)
            if (j < K - 1) {
                p = __builtin_fmaf(w[(long long)d * K + j], (float)old[j], p);
                if (j > 0)
                    st[j - 1] = old[j];
            }
        p = __builtin_fmaf(w[(long long)d * K + K - 1], (float)in, p);
        if (K > 1)
            st[K - 2] = in;
        *out = (E)(silu_on ? silu(p) : p);
    }
}

// ---- host ------------------------------------------------------------------------

// Tiles of `v` elements over rows of L: threads along a row, and tiles along it.
struct Tiling {
    int txl;
    long long along;
};
inline Tiling tiling(int L, int v) {
    const long long nb = L > 0 ? cdivll(L, v) : 1;
    Tiling t = {0, 0};
    while (t.txl < 8 && (1ll << t.txl) < nb)
        ++t.txl;
    t.along = cdivll(nb, 1ll << t.txl);
    return t;
}

// Parts of a channel's (row, tile) pairs: eight waves a SIMD over the card where
// there are that many pairs.
constexpr int kBlocks = 2048;
inline long long most_parts(int D) { return cdivll(kBlocks, D); }

inline bool conv_shape(int type, int B, int D, int L, int K) {
    return type_size(type) && B >= 0 && D >= 1 && L >= 0 && L < (1 << 30) && K >= 1 &&
           K <= FINC_MAX_TAPS && (long long)B * D < (1ll << 31) - 256;
}

template <typename E, bool SILU, bool BACK>
void launch_taps(int K, const ConvArgs &c, dim3 grid, hipStream_t s) {
#define FINC_TAPS(k)                                                                         \
    case k:                                                                                  \
        if (BACK)                                                                            \
            hipLaunchKernelGGL((conv_backward_kernel<E, k, SILU>), grid, dim3(kThreads), 0,  \
                               s, c);                                                        \
        else                                                                                 \
            hipLaunchKernelGGL((conv_forward_kernel<E, k, SILU>), grid, dim3(kThreads), 0, s, \
                               c);                                                           \
        break;
    switch (K) {
        FINC_TAPS(1)
        FINC_TAPS(2)
        FINC_TAPS(3)
        FINC_TAPS(4)
        FINC_TAPS(5)
        FINC_TAPS(6)
        FINC_TAPS(7)
        FINC_TAPS(8)
    }
#undef FINC_TAPS
}

// The fields that both directions share; FINC_OK, or the error.
int conv_common(const finc_conv_args *a, bool back, ConvArgs &c) {
    c = ConvArgs{};
    c.x = a->x.p;
    c.xb = a->x.sb;
    c.xd = a->x.sd;
    c.w = a->w;
    c.bias = a->bias;
    c.state = a->state;
    c.lengths = a->lengths;
    c.B = a->B;
    c.D = a->D;
    c.L = a->L;
    const Tiling t = tiling(a->L, kTileBytes(back) / type_size(a->type));
    c.txl = t.txl;
    if (t.along >= (1ll << 31))
        return FINC_EUNSUPPORTED;
    c.tiles_t = (int)t.along;
    c.div_d = make_fastdiv(a->D);
    c.div_t = make_fastdiv(c.tiles_t);
    return FINC_OK;
}

}  // namespace

extern "C" {

int finc_causal_conv_forward(const finc_conv_args *a, hipStream_t stream) {
    if (!a || !conv_shape(a->type, a->B, a->D, a->L, a->K))
        return FINC_EINVAL;
    const int sz = type_size(a->type);
    const long long st = (long long)a->B * a->D * (a->K - 1);
    const Region in[] = {raster(a->x, a->B, a->D, a->L, sz), flat(a->w, (long long)a->D * a->K, 4),
                         flat(a->bias, a->bias ? a->D : 0, 4),
                         flat(a->state, a->state ? st : 0, sz),
                         flat(a->lengths, a->lengths ? a->B : 0, 4)};
    const Region out[] = {raster(a->y, a->B, a->D, a->L, sz),
                          flat(a->state_out, a->state_out ? st : 0, sz)};
    for (const Region &r : in)
        if (!readable(r))
            return FINC_EINVAL;
    for (const Region &r : out)
        if (!writable(r))
            return FINC_EINVAL;
    if (!disjoint(in, out))
        return FINC_EINVAL;
    if (a->B == 0)
        return FINC_OK;
    ConvArgs c;
    const int rc = conv_common(a, false, c);
    if (rc != FINC_OK)
        return rc;
    c.y = a->y.p;
    c.yb = a->y.sb;
    c.yd = a->y.sd;
    c.state_out = a->state_out;
    const long long rows = cdivll((long long)a->B * a->D, kThreads >> c.txl);
    if (rows * c.tiles_t >= (1ll << 31))
        return FINC_EUNSUPPORTED;
    with_type(a->type, [&](auto e) {
        typedef decltype(e) E;
        const dim3 grid = grid_of(rows * c.tiles_t);
        if (a->silu)
            launch_taps<E, true, false>(a->K, c, grid, stream);
        else
            launch_taps<E, false, false>(a->K, c, grid, stream);
    });
    return launched();
}

size_t finc_causal_conv_workspace_bytes(int B, int D, int L, int K) {
    if (!conv_shape(FINC_F32, B, D, L, K))
        return 0;
    return (size_t)((most_parts(D) * D * (K + 1) * 4 + 255) / 256 * 256);
}

int finc_causal_conv_backward(const finc_conv_args *a, const finc_conv_grads *g,
                              hipStream_t stream) {
    if (!a || !g || !conv_shape(a->type, a->B, a->D, a->L, a->K) || !g->dw ||
        ((uintptr_t)g->workspace & 255u))
        return FINC_EINVAL;
    const int sz = type_size(a->type), B = a->B, D = a->D, L = a->L, K = a->K;
    const long long st = (long long)B * D * (K - 1);
    const Region in[] = {raster(a->x, B, D, L, sz), raster(g->dy, B, D, L, sz),
                         flat(a->w, (long long)D * K, 4), flat(a->bias, a->bias ? D : 0, 4),
                         flat(a->state, a->state ? st : 0, sz),
                         flat(g->dstate_out, g->dstate_out ? st : 0, sz),
                         flat(a->lengths, a->lengths ? B : 0, 4)};
    const Region out[] = {raster(g->dx, B, D, L, sz), flat(g->dw, (long long)D * K, 4),
                          flat(g->dbias, g->dbias ? D : 0, 4),
                          flat(g->dstate, g->dstate ? st : 0, sz),
                          flat(g->workspace, (long long)finc_causal_conv_workspace_bytes(B, D, L, K), 1)};
    for (const Region &r : in)
        if (!readable(r))
            return FINC_EINVAL;
    for (const Region &r : out)
        if (!writable(r))
            return FINC_EINVAL;
    if (!disjoint(in, out))
        return FINC_EINVAL;
    ConvArgs c;
    const int rc = conv_common(a, true, c);
    if (rc != FINC_OK)
        return rc;
    c.dy = g->dy.p;
    c.gb = g->dy.sb;
    c.gd = g->dy.sd;
    c.dx = g->dx.p;
    c.ob = g->dx.sb;
    c.od = g->dx.sd;
    c.dstate = g->dstate;
    c.dstate_out = g->dstate_out;
    c.partial = (float *)g->workspace;
    const long long rows = cdivll(B, kThreads >> c.txl);
    if (rows * c.tiles_t >= (1ll << 31) - kBlocks)
        return FINC_EUNSUPPORTED;
    c.tiles_r = (int)rows;
    const long long units = rows * c.tiles_t, most = most_parts(D);
    c.parts = (int)(units < most ? units : most);
    if (c.parts > 0) {
        with_type(a->type, [&](auto e) {
            typedef decltype(e) E;
            const dim3 grid = grid_of((long long)D * c.parts);
            if (a->silu)
                launch_taps<E, true, true>(K, c, grid, stream);
            else
                launch_taps<E, false, true>(K, c, grid, stream);
        });
        const int r2 = launched();
        if (r2 != FINC_OK)
            return r2;
    }
    hipLaunchKernelGGL(conv_sum_kernel, grid_of(cdivll((long long)D * (K + 1), 32)), dim3(256), 0,
                       stream, c.partial, c.parts, g->dw, g->dbias, D, K);
    return launched();
}

int finc_causal_conv_step(int type, const void *x, long long sx, void *y, long long sy,
                          const float *w, const float *bias, void *state, const int *slots, int B,
                          int S, int D, int K, int silu, hipStream_t stream) {
    if (!conv_shape(type, B, D, 1, K) || S < 0 || (!slots && S < B))
        return FINC_EINVAL;
    const int sz = type_size(type);
    const long long st = elements(S, D, K - 1);
    const Region in[] = {{x, B, sx, 1, 0, D, sz}, flat(w, (long long)D * K, 4),
                         flat(bias, bias ? D : 0, 4), flat(slots, slots ? B : 0, 4)};
    const Region out[] = {{y, B, sy, 1, 0, D, sz}, flat(state, st, sz)};
    for (const Region &r : in)
        if (!readable(r))
            return FINC_EINVAL;
    for (const Region &r : out)
        if (!writable(r))
            return FINC_EINVAL;
    if (!disjoint(in, out))
        return FINC_EINVAL;
    if (B == 0)
        return FINC_OK;
    with_type(type, [&](auto e) {
        typedef decltype(e) E;
        hipLaunchKernelGGL(conv_step_kernel<E>,
                           dim3((unsigned)cdivll(D, kThreads), (unsigned)(B < 32768 ? B : 32768)),
                           dim3(kThreads), 0, stream, (const E *)x, sx, (E *)y, sy, w, bias,
                           (E *)state, slots, B, S, D, K, silu);
    });
    return launched();
}

}  // extern "C"
