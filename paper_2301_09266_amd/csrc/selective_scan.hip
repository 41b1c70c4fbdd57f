// selective_scan.hip -- the selective state space scan, its gradients and its
// single-position form (finc_selective_scan_* of finc.h).
//
//   h_t = a_t h_{t-1} + b_t,  a_t = exp(delta_t A_n),  b_t = delta_t x_t B_t,n,
//   y_t = sum_n C_t,n h_t + Dskip x_t  for every channel and its N states.
//
// A row of 16 lanes holds one channel's positions, T neighbours a lane.  A lane
// composes its T maps h -> a h + b into one, a scan over the row's lanes composes
// the lanes before it (the map of a lane's whole run is exp(A sum delta), one
// exponential), and a second pass over the T positions, from the state that the
// scan gives, reads the same a from registers: each (position, state) takes one
// exponential, and 5 multiplies and multiply-adds.  Those bound the scan: at N = 16 in
// bf16 a position's 8 bytes of activations take 1/4 of their time.  Rows walk the
// raster in parts of 16 T positions with the state in LDS between them.
#include "seq_common.h"

namespace {

using namespace finc_seq;

constexpr int kThreads = 256;
constexpr float kLog2e = 1.44269504088896341f;

struct Rows {
    void *p;
    long long sb, sd;
    template <typename E>
    __device__ E *row(int b, long long d) const {
        return (E *)p + (b * sb + d * sd);
    }
};
inline Rows rows_of(const finc_raster &r) { return {r.p, r.sb, r.sd}; }

struct ScanArgs {
    Rows x, dt, z, Bm, Cm, y;
    const float *A, *Dskip, *dt_bias, *state;
    float *state_out, *states;
    const int *lengths;
    int B, D, L, N, G, Dg;   // Dg: channels of a group
    int softplus, parts;     // parts: of 16 T positions, of the whole raster
    int blocks;              // of channels, in a group
};

// ---- the scan over a row's lanes ---------------------------------------------------
// (a, h) of the lane's own run -> of the row's lanes up to it, for S states side by
// side.  A DPP operand needs two wait states after the instruction that wrote it:
// with one state there is a gap between uses, with more the other states fill it.
// A lane whose source lies outside the row keeps its value.

#define FINC_STEP1(ctl)                                                                     \
    "v_fmac_f32_dpp %1, %1, %0 " ctl " row_mask:0xf bank_mask:0xf\n"                        \
    "v_mul_f32_dpp %0, %0, %0 " ctl " row_mask:0xf bank_mask:0xf\n"                         \
    "s_nop 0\n"
#define FINC_STEP2(ctl)                                                                     \
    "v_fmac_f32_dpp %1, %1, %0 " ctl " row_mask:0xf bank_mask:0xf\n"                        \
    "v_fmac_f32_dpp %3, %3, %2 " ctl " row_mask:0xf bank_mask:0xf\n"                        \
    "v_mul_f32_dpp %0, %0, %0 " ctl " row_mask:0xf bank_mask:0xf\n"                         \
    "v_mul_f32_dpp %2, %2, %2 " ctl " row_mask:0xf bank_mask:0xf\n"

__device__ inline void scan_up(float (&a)[1], float (&h)[1]) {
    asm volatile("s_nop 1\n" FINC_STEP1("row_shr:1") FINC_STEP1("row_shr:2") FINC_STEP1(
                     "row_shr:4") FINC_STEP1("row_shr:8") "s_nop 1"
                 : "+v"(a[0]), "+v"(h[0]));
}
__device__ inline void scan_up(float (&a)[2], float (&h)[2]) {
    asm volatile("s_nop 1\n" FINC_STEP2("row_shr:1") FINC_STEP2("row_shr:2") FINC_STEP2(
                     "row_shr:4") FINC_STEP2("row_shr:8") "s_nop 1"
                 : "+v"(a[0]), "+v"(h[0]), "+v"(a[1]), "+v"(h[1]));
}
// The same towards the row's first lane.
__device__ inline void scan_down(float (&a)[1], float (&h)[1]) {
    asm volatile("s_nop 1\n" FINC_STEP1("row_shl:1") FINC_STEP1("row_shl:2") FINC_STEP1(
                     "row_shl:4") FINC_STEP1("row_shl:8") "s_nop 1"
                 : "+v"(a[0]), "+v"(h[0]));
}

// The neighbour's value; `edge` where the row has none.
template <int CTRL>
__device__ inline float neighbour(float edge, float v) {
    return __builtin_bit_cast(
        float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, edge),
                                           __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}
constexpr int kFromLower = 0x111, kFromUpper = 0x101;   // row_shr:1, row_shl:1

__device__ inline int row_length(const int *lengths, int b, int L) {
    return lengths ? min(max(lengths[b], 0), L) : L;
}

// A part's tile of B or C in LDS: position q of state n, fp32, four neighbours
// together and the row's lanes side by side, so that the 16 lanes of a row read 256
// neighbouring bytes (the other rows read the same ones).
template <int T>
__device__ inline int tile_at(int n, int j4, int lane) {
    return ((n * (T / 4) + j4) * 16 + lane) * 4;
}

template <int S>
struct Out {
    float h[S];
};

// S states of a row's part: adds C h to y and gives the state at the part's end in
// the row's last lane; `in` are the states before the part.
template <int T, int S>
__device__ inline Out<S> scan_states(const float *tb, const float *tc, const int (&n)[S],
                                     const float (&A2)[S], const float (&in)[S], int lane,
                                     const float (&delta)[T], const float (&dx)[T], float sum,
                                     float (&y)[T], float (&start)[S]) {
    float a[S][T], h[S], m[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        h[s] = 0.0f;
#pragma unroll
        for (int j4 = 0; j4 < T / 4; ++j4) {
            const float4 b = *(const float4 *)(tb + tile_at<T>(n[s], j4, lane));
            const float bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = 4 * j4 + i;
                a[s][j] = __builtin_amdgcn_exp2f(A2[s] * delta[j]);
                h[s] = __builtin_fmaf(a[s][j], h[s], dx[j] * bv[i]);
            }
        }
        m[s] = __builtin_amdgcn_exp2f(A2[s] * sum);
    }
    scan_up(m, h);
    Out<S> end;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        end.h[s] = __builtin_fmaf(m[s], in[s], h[s]);
        float g = start[s] = neighbour<kFromLower>(in[s], end.h[s]);
#pragma unroll
        for (int j4 = 0; j4 < T / 4; ++j4) {
            const float4 b = *(const float4 *)(tb + tile_at<T>(n[s], j4, lane));
            const float4 c = *(const float4 *)(tc + tile_at<T>(n[s], j4, lane));
            const float bv[4] = {b.x, b.y, b.z, b.w}, cv[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = 4 * j4 + i;
                g = __builtin_fmaf(a[s][j], g, dx[j] * bv[i]);
                y[j] = __builtin_fmaf(cv[i], g, y[j]);
            }
        }
    }
    return end;
}

// One block: CB = 16 / W channels of one batch row and group, W waves sharing a
// channel's states (each N / W of them) where there are few channels.
template <typename E, int T, int W>
__global__ __launch_bounds__(kThreads) void scan_forward_kernel(ScanArgs a) {
    constexpr int CB = 16 / W, P = 16 * T;   // P: positions of a part
    extern __shared__ __attribute__((aligned(16))) float lds[];
    float *tb = lds, *tc = tb + a.N * P;
    float *hs = tc + a.N * P;                // the states between parts, CB x N
    float *As = hs + CB * a.N;               // A log2 e, CB x N
    float *red = As + CB * a.N;              // W > 1: the waves' sums of y
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 15, rowi = (tid >> 4) & 3;
    int blk = blockIdx.x;
    const int cb = blk % a.blocks;
    blk /= a.blocks;
    const int grp = blk % a.G, b = blk / a.G;
    const int split = wave % W, cl = (wave / W) * 4 + rowi;   // channel in the block
    const int dg = cb * CB + cl;
    const bool live = dg < a.Dg;
    const int d = grp * a.Dg + (live ? dg : 0);
    const int n_pos = row_length(a.lengths, b, a.L);
    for (int i = tid; i < CB * a.N; i += kThreads) {
        const int c = i / a.N, n = i - c * a.N, dd = cb * CB + c;
        const bool ok = dd < a.Dg;
        const long long at = (long long)(grp * a.Dg + (ok ? dd : 0)) * a.N + n;
        As[i] = ok ? a.A[at] * kLog2e : 0.0f;
        hs[i] = ok && a.state ? a.state[(long long)b * a.D * a.N + at] : 0.0f;
    }
    const float bias = a.dt_bias ? a.dt_bias[d] : 0.0f;
    const float skip = a.Dskip ? a.Dskip[d] : 0.0f;
    const E *xr = a.x.row<const E>(b, d), *dr = a.dt.row<const E>(b, d);
    const E *zr = a.z.p ? a.z.row<const E>(b, d) : nullptr;
    E *yr = a.y.row<E>(b, d);
    const int parts = (n_pos + P - 1) / P;
    for (int part = 0; part < parts; ++part) {
        const int p0 = part * P, t0 = p0 + lane * T;
        // positions past the row's length: delta 0 keeps the state, B and C are 0
        for (int u = tid; u < 2 * a.N * (P / 4); u += kThreads) {
            const int which = u >= a.N * (P / 4), v = u - which * a.N * (P / 4);
            const int n = v / (P / 4), q = v - n * (P / 4);
            float t[4];
            load_upto<E, 4>((which ? a.Cm : a.Bm).row<const E>(b, grp * a.N + n) + p0 + 4 * q,
                            n_pos - p0 - 4 * q, t);
            *(float4 *)((which ? tc : tb) + tile_at<T>(n, q % (T / 4), q / (T / 4))) =
                make_float4(t[0], t[1], t[2], t[3]);
        }
        float x[T], delta[T], dx[T], y[T];
        load_upto<E, T>(xr + t0, live ? n_pos - t0 : 0, x);
        load_upto<E, T>(dr + t0, live ? n_pos - t0 : 0, delta);
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < T; ++j) {
            float v = delta[j] + bias;
            if (a.softplus)
                v = softplus(v);
            delta[j] = live && t0 + j < n_pos ? v : 0.0f;
            dx[j] = delta[j] * x[j];
            sum += delta[j];
            y[j] = 0.0f;
        }
        __syncthreads();
        for (int i = split; i < a.N; i += W) {
            const int n[1] = {i};
            const float A2[1] = {As[cl * a.N + i]}, in[1] = {hs[cl * a.N + i]};
            float start[1];
            const Out<1> end =
                scan_states<T, 1>(tb, tc, n, A2, in, lane, delta, dx, sum, y, start);
            if (a.states && live && lane == 0)
                a.states[(((long long)b * a.D + d) * a.parts + part) * a.N + i] = in[0];
            if (lane == 15)
                hs[cl * a.N + i] = end.h[0];
        }
        if (W > 1) {
            float4 *r = (float4 *)red;
#pragma unroll
            for (int j4 = 0; j4 < T / 4; ++j4)
                r[(wave * (T / 4) + j4) * 64 + (tid & 63)] =
                    make_float4(y[4 * j4], y[4 * j4 + 1], y[4 * j4 + 2], y[4 * j4 + 3]);
            __syncthreads();
            if (split == 0) {
#pragma unroll
                for (int w = 1; w < W; ++w)
#pragma unroll
                    for (int j4 = 0; j4 < T / 4; ++j4) {
                        const float4 v = r[((wave + w) * (T / 4) + j4) * 64 + (tid & 63)];
                        y[4 * j4] += v.x;
                        y[4 * j4 + 1] += v.y;
                        y[4 * j4 + 2] += v.z;
                        y[4 * j4 + 3] += v.w;
                    }
            }
        }
        if (split == 0 && live) {
            float z[T];
            if (zr)
                load_upto<E, T>(zr + t0, n_pos - t0, z);
#pragma unroll
            for (int j = 0; j < T; ++j) {
                y[j] = __builtin_fmaf(skip, x[j], y[j]);
                if (zr)
                    y[j] *= silu(z[j]);
                if (t0 + j >= n_pos)
                    y[j] = 0.0f;
            }
            store_upto<E, T>(yr + t0, a.L - t0, y);
        }
        __syncthreads();
    }
    // padding
    for (int c = 0; c < CB; ++c) {
        const int dd = cb * CB + c;
        if (dd >= a.Dg)
            break;
        E *r = a.y.row<E>(b, grp * a.Dg + dd);
        for (long long t = (long long)parts * P + tid; t < a.L; t += kThreads)
            r[t] = (E)0.0f;
    }
    __syncthreads();
    if (a.state_out)
        for (int i = tid; i < CB * a.N; i += kThreads) {
            const int c = i / a.N, n = i - c * a.N, dd = cb * CB + c;
            if (dd < a.Dg)
                a.state_out[((long long)b * a.D + grp * a.Dg + dd) * a.N + n] = hs[i];
        }
}

// ---- gradients ----------------------------------------------------------------------
// With G_t = a_t g_t the gradient of the state obeys g_t = C_t dy_t + G_{t+1}: the
// same scan towards lower positions.  A workgroup owns a set of channels of one batch
// row and walks the parts from the last to the first; within a part it takes 4 H
// channels at a time.  W waves share the states of four channels, four states a wave
// and a channel a row of 16 lanes, so that a wave keeps B, C and their gradients of
// its four states in registers while the channels pass: dB and dC are sums over the
// channels, and reach memory once a set.  The states inside a part are recomputed from
// the one that the forward kept at its start.

struct GradArgs {
    ScanArgs f;
    Rows dy, dx, ddt, dz;
    const float *dstate_out;
    float *dstate;
    float *shared;    // dB then dC by sets, (2, sets, B, G N, L)
    float *params;    // dA, dDskip, ddt_bias by batch rows, (B, D (N + 2))
    int set, sets;    // channels of a set, sets of a group
};

template <int T>
__device__ inline int slot_at(int t) {
    return ((t % T / 4) * 16 + t / T) * 4 + t % 4;
}

// Positions of one channel that a thread prepares and finishes.
template <int T, int W>
constexpr int kItems = T / W > 1 ? T / W : 1;

inline size_t backward_lds(int N, int T, int W, int H, int set) {
    return ((size_t)3 * 4 * H * 16 * T + (size_t)3 * T * 64 * W * H + (size_t)3 * set * N +
            (size_t)set * W * 2) * 4;
}

template <typename E, int T, int W, int H>
__global__ __launch_bounds__(64 * W * H) void scan_backward_kernel(GradArgs ga) {
    constexpr int P = 16 * T, CB = 4 * H, TH = 64 * W * H, I = kItems<T, W>;
    const ScanArgs &a = ga.f;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    float *pre = lds;                              // delta, delta x, dy of CB channels
    float *sums = pre + 3 * CB * P;                // the waves' sums over their states
    float *carry = sums + 3 * T * 64 * W * H;      // G at the part's end, set x N
    float *As = carry + ga.set * a.N;              // A log2 e
    float *dAs = As + ga.set * a.N;                // dA
    float *ps = dAs + ga.set * a.N;                // dDskip, ddt_bias: set x W rows x 2
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 15, rowi = (tid >> 4) & 3;
    const int w = wave % W, half = wave / W, n0 = 4 * w;
    int blk = blockIdx.x;
    const int set = blk % ga.sets;
    blk /= ga.sets;
    const int grp = blk % a.G, b = blk / a.G;
    const int c0 = set * ga.set;                   // the set's first channel in the group
    const int count = min(ga.set, a.Dg - c0);
    const long long first = (long long)grp * a.Dg + c0;
    const int n_pos = row_length(a.lengths, b, a.L);
    const int parts = (n_pos + P - 1) / P;
    for (int i = tid; i < ga.set * a.N; i += TH) {
        const bool ok = i < count * a.N;
        As[i] = ok ? a.A[first * a.N + i] * kLog2e : 0.0f;
        carry[i] = ok && ga.dstate_out ? ga.dstate_out[((long long)b * a.D + first) * a.N + i] : 0.0f;
        dAs[i] = 0.0f;
    }
    for (int i = tid; i < ga.set * W * 2; i += TH)
        ps[i] = 0.0f;
    __syncthreads();
    for (int part = parts - 1; part >= 0; --part) {
        const int p0 = part * P;
        float Bv[4][T], Cv[4][T], dB[4][T], dC[4][T];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const bool ok = n0 + s < a.N;
            const long long r = (long long)grp * a.N + (ok ? n0 + s : 0);
            const int left = ok ? n_pos - p0 - lane * T : 0;
            load_upto<E, T>(a.Bm.row<const E>(b, r) + p0 + lane * T, left, Bv[s]);
            load_upto<E, T>(a.Cm.row<const E>(b, r) + p0 + lane * T, left, Cv[s]);
#pragma unroll
            for (int j = 0; j < T; ++j)
                dB[s][j] = dC[s][j] = 0.0f;
        }
        for (int cb = 0; cb < count; cb += CB) {
            // what a position needs, once a channel: I neighbours a thread
            const int at = tid * I, cq = at / P, pos = at - cq * P;
            const bool mine = cq < CB, live = mine && cb + cq < count;
            const int d = (int)first + (live ? cb + cq : 0);
            float x[I], delta[I], slope[I], z[I], dout[I], dy[I];
            const int left = live ? n_pos - p0 - pos : 0;
            load_upto<E, I>(a.x.row<const E>(b, d) + p0 + pos, left, x);
            load_upto<E, I>(a.dt.row<const E>(b, d) + p0 + pos, left, delta);
            load_upto<E, I>(ga.dy.row<const E>(b, d) + p0 + pos, left, dout);
            if (a.z.p)
                load_upto<E, I>(a.z.row<const E>(b, d) + p0 + pos, left, z);
            const float bias = a.dt_bias ? a.dt_bias[d] : 0.0f;
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const float v = delta[i] + bias;
                slope[i] = a.softplus ? sigmoid(v) : 1.0f;
                delta[i] = i < left ? (a.softplus ? softplus(v) : v) : 0.0f;
                dy[i] = a.z.p ? dout[i] * silu(z[i]) : dout[i];
            }
            if (mine) {
                float *q = pre + cq * P;
#pragma unroll
                for (int i = 0; i < I; ++i) {
                    q[slot_at<T>(pos + i)] = delta[i];
                    q[CB * P + slot_at<T>(pos + i)] = delta[i] * x[i];
                    q[2 * CB * P + slot_at<T>(pos + i)] = dy[i];
                }
            }
            __syncthreads();
            {
                const int ch = half * 4 + rowi;                 // of the CB channels
                const int cs = min(cb + ch, ga.set - 1);        // in the set
                const bool here = cb + ch < count;
                const float *q = pre + ch * P + lane * 4;
                float de[T], dx[T], g[T], gB[T], sA[T], yv[T], sum = 0.0f;
#pragma unroll
                for (int j4 = 0; j4 < T / 4; ++j4) {
                    const float4 u = *(const float4 *)(q + j4 * 64);
                    const float4 v = *(const float4 *)(q + CB * P + j4 * 64);
                    const float4 e = *(const float4 *)(q + 2 * CB * P + j4 * 64);
                    const float uu[4] = {u.x, u.y, u.z, u.w}, vv[4] = {v.x, v.y, v.z, v.w};
                    const float ee[4] = {e.x, e.y, e.z, e.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int j = 4 * j4 + i;
                        de[j] = uu[i];
                        dx[j] = vv[i];
                        g[j] = ee[i];
                        sum += uu[i];
                        gB[j] = sA[j] = yv[j] = 0.0f;
                    }
                }
                const float *st =
                    a.states + (((long long)b * a.D + first + (here ? cb + ch : 0)) * a.parts +
                                part) * a.N;
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const int n = n0 + s;
                    if (n >= a.N)   // the same in the whole wave
                        break;
                    const float A2 = As[cs * a.N + n], in = here ? st[n] : 0.0f;
                    const float after = carry[cs * a.N + n];
                    float av[T], h[T], m[1], e[1] = {0.0f};
#pragma unroll
                    for (int j = 0; j < T; ++j) {
                        av[j] = __builtin_amdgcn_exp2f(A2 * de[j]);
                        e[0] = __builtin_fmaf(av[j], e[0], dx[j] * Bv[s][j]);
                    }
                    const float run = m[0] = __builtin_amdgcn_exp2f(A2 * sum);
                    scan_up(m, e);
                    const float start =
                        neighbour<kFromLower>(in, __builtin_fmaf(m[0], in, e[0]));
                    float prev = start;
#pragma unroll
                    for (int j = 0; j < T; ++j)
                        prev = h[j] = __builtin_fmaf(av[j], prev, dx[j] * Bv[s][j]);
                    // G below the lane's run, from 0 above it, then from the lanes above
                    e[0] = 0.0f;
#pragma unroll
                    for (int j = T - 1; j >= 0; --j)
                        e[0] = av[j] * __builtin_fmaf(Cv[s][j], g[j], e[0]);
                    m[0] = run;
                    scan_down(m, e);
                    const float low = __builtin_fmaf(m[0], after, e[0]);
                    float G = neighbour<kFromUpper>(after, low), dA = 0.0f;
#pragma unroll
                    for (int j = T - 1; j >= 0; --j) {
                        const float gt = __builtin_fmaf(Cv[s][j], g[j], G);
                        G = av[j] * gt;
                        dC[s][j] = __builtin_fmaf(g[j], h[j], dC[s][j]);
                        dB[s][j] = __builtin_fmaf(gt, dx[j], dB[s][j]);
                        gB[j] = __builtin_fmaf(gt, Bv[s][j], gB[j]);
                        yv[j] = __builtin_fmaf(Cv[s][j], h[j], yv[j]);
                        const float t = G * (j ? h[j ? j - 1 : 0] : start);
                        sA[j] = __builtin_fmaf(A2, t, sA[j]);
                        dA = __builtin_fmaf(de[j], t, dA);
                    }
                    dA = row_sum(dA);
                    if (here) {
                        if (lane == 15)
                            dAs[cs * a.N + n] += dA;
                        if (lane == 0)
                            carry[cs * a.N + n] = low;
                    }
                }
                float4 *o = (float4 *)sums + (wave * 3 * (T / 4)) * 64 + (tid & 63);
#pragma unroll
                for (int j4 = 0; j4 < T / 4; ++j4) {
                    const int j = 4 * j4;
                    o[j4 * 64] = make_float4(gB[j], gB[j + 1], gB[j + 2], gB[j + 3]);
                    o[(T / 4 + j4) * 64] = make_float4(sA[j], sA[j + 1], sA[j + 2], sA[j + 3]);
                    o[(2 * (T / 4) + j4) * 64] =
                        make_float4(yv[j], yv[j + 1], yv[j + 2], yv[j + 3]);
                }
            }
            __syncthreads();
            // the gradients of the positions that this thread prepared
            float sD = 0.0f, sb = 0.0f;
            if (live) {
                const float skip = a.Dskip ? a.Dskip[d] : 0.0f;
                float ox[I], ot[I], oz[I];
#pragma unroll
                for (int i = 0; i < I; ++i) {
                    const int t = pos + i, ln = (cq & 3) * 16 + t / T, j = t % T;
                    const float *s0 = sums + (((cq >> 2) * W * 3 * (T / 4) + j / 4) * 64 + ln) * 4 +
                                      j % 4;
                    float v[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int k = 0; k < W; ++k)
#pragma unroll
                        for (int kind = 0; kind < 3; ++kind)
                            v[kind] += s0[((k * 3 + kind) * (T / 4)) * 256];
                    const bool in = i < left;
                    const float dd = x[i] * v[0] + v[1] * 0.693147180559945309f;
                    ot[i] = in ? dd * slope[i] : 0.0f;
                    ox[i] = in ? __builtin_fmaf(delta[i], v[0], skip * dy[i]) : 0.0f;
                    sb += ot[i];
                    sD = __builtin_fmaf(dy[i], x[i], sD);
                    if (a.z.p) {
                        const float y = __builtin_fmaf(skip, x[i], v[2]);
                        oz[i] = in ? dout[i] * y * silu_grad(z[i], sigmoid(z[i])) : 0.0f;
                    }
                }
                const int room = a.L - p0 - pos;
                store_upto<E, I>(ga.dx.row<E>(b, d) + p0 + pos, room, ox);
                store_upto<E, I>(ga.ddt.row<E>(b, d) + p0 + pos, room, ot);
                if (a.z.p)
                    store_upto<E, I>(ga.dz.row<E>(b, d) + p0 + pos, room, oz);
            }
            sD = row_sum(sD);
            sb = row_sum(sb);
            if (live && lane == 15) {
                // the channel's P / I threads are P / I / 16 rows
                float *q = ps + ((cb + cq) * W + (pos / I) / 16) * 2;
                q[0] += sD;
                q[1] += sb;
            }
        }
        // dB and dC of the part: the rows, then the halves
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int j = 0; j < T; ++j) {
                dB[s][j] += __shfl_xor(dB[s][j], 16, 64);
                dB[s][j] += __shfl_xor(dB[s][j], 32, 64);
                dC[s][j] += __shfl_xor(dC[s][j], 16, 64);
                dC[s][j] += __shfl_xor(dC[s][j], 32, 64);
            }
        // sums is free once every thread has finished its positions
        __syncthreads();
        if (H > 1) {
            if (half > 0 && rowi == 0)
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    store_vec<float, T>(sums + ((wave * 8 + s) * 16 + lane) * T, dB[s]);
                    store_vec<float, T>(sums + ((wave * 8 + 4 + s) * 16 + lane) * T, dC[s]);
                }
            __syncthreads();
        }
        if (half == 0 && rowi == 0) {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                if (n0 + s >= a.N)
                    break;
#pragma unroll
                for (int k = 1; k < H; ++k) {
                    float u[T], v[T];
                    load_vec<float, T>(sums + (((k * W + w) * 8 + s) * 16 + lane) * T, u);
                    load_vec<float, T>(sums + (((k * W + w) * 8 + 4 + s) * 16 + lane) * T, v);
#pragma unroll
                    for (int j = 0; j < T; ++j) {
                        dB[s][j] += u[j];
                        dC[s][j] += v[j];
                    }
                }
                const long long rows = (long long)a.G * a.N;
                const long long r =
                    ((long long)set * a.B + b) * rows + (long long)grp * a.N + n0 + s;
                const int t0 = p0 + lane * T;
                store_upto<float, T>(ga.shared + r * a.L + t0, a.L - t0, dB[s]);
                store_upto<float, T>(ga.shared + ((long long)ga.sets * a.B * rows + r) * a.L + t0,
                                     a.L - t0, dC[s]);
            }
        }
        __syncthreads();
    }
    __syncthreads();
    // padding
    for (int c = 0; c < count; ++c)
        for (long long t = (long long)parts * P + tid; t < a.L; t += TH) {
            ga.dx.row<E>(b, (int)first + c)[t] = (E)0.0f;
            ga.ddt.row<E>(b, (int)first + c)[t] = (E)0.0f;
            if (a.z.p)
                ga.dz.row<E>(b, (int)first + c)[t] = (E)0.0f;
        }
    float *out = ga.params + (long long)b * a.D * (a.N + 2);
    for (int i = tid; i < count * a.N; i += TH) {
        out[first * a.N + i] = dAs[i];
        if (ga.dstate)
            ga.dstate[((long long)b * a.D + first) * a.N + i] = carry[i];
    }
    for (int c = tid; c < count; c += TH) {
        float sD = 0.0f, sb = 0.0f;
        for (int k = 0; k < W; ++k) {
            sD += ps[(c * W + k) * 2];
            sb += ps[(c * W + k) * 2 + 1];
        }
        out[(long long)a.D * a.N + first + c] = sD;
        out[(long long)a.D * (a.N + 1) + first + c] = sb;
    }
}

// dB and dC: the sets' sums in order.
template <typename E>
__global__ __launch_bounds__(256) void shared_sum_kernel(GradArgs ga, Rows dB, Rows dC) {
    const ScanArgs &a = ga.f;
    const int rows = a.G * a.N;
    const long long tiles = (a.L + 1023) / 1024;
    long long blk = blockIdx.x;
    const long long tile = blk % tiles;
    blk /= tiles;
    const int r = (int)(blk % rows);
    blk /= rows;
    const int b = (int)(blk % a.B), which = (int)(blk / a.B);
    const int t0 = (int)(tile * 1024 + threadIdx.x * 4);
    if (t0 >= a.L)
        return;
    const int n_pos = row_length(a.lengths, b, a.L);
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const long long step = (long long)a.B * rows * a.L;
    const float *p = ga.shared + which * ga.sets * step + ((long long)b * rows + r) * a.L + t0;
    for (int k = 0; k < ga.sets; ++k) {
        float v[4];
        load_upto<float, 4>(p + k * step, n_pos - t0, v);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            s[i] += v[i];
    }
    store_upto<E, 4>((which ? dC : dB).row<E>(b, r) + t0, a.L - t0, s);
}

// dA, dDskip, ddt_bias: the batch rows' sums, eight groups in turn, then in order.
__global__ __launch_bounds__(256) void param_sum_kernel(GradArgs ga, float *dA, float *dD,
                                                        float *db) {
    __shared__ float red[8][33];
    const ScanArgs &a = ga.f;
    const long long n = (long long)a.D * (a.N + 2);
    const int l = threadIdx.x & 31, g = threadIdx.x >> 5;
    const long long i = blockIdx.x * 32ll + l;
    float s = 0.0f;
    if (i < n)
        for (int b = g; b < a.B; b += 8)
            s += ga.params[b * n + i];
    red[g][l] = s;
    __syncthreads();
    if (g || i >= n)
        return;
    s = 0.0f;
    for (int k = 0; k < 8; ++k)
        s += red[k][l];
    const long long nA = (long long)a.D * a.N;
    if (i < nA)
        dA[i] = s;
    else if (i < nA + a.D) {
        if (dD)
            dD[i - nA] = s;
    } else if (db)
        db[i - nA - a.D] = s;
}

// ---- one position ---------------------------------------------------------------

struct StepArgs {
    const void *x, *dt, *z, *Bm, *Cm;
    void *y;
    const float *A, *Dskip, *dt_bias;
    float *state;
    const int *slots;
    long long sx, sdt, sz, sB, sC, sy;
    int B, S, D, N, G, Dg, softplus;
};

// Q lanes a channel, four states each at a time.
template <typename E, int Q>
__global__ __launch_bounds__(kThreads) void scan_step_kernel(StepArgs a) {
    const int q = threadIdx.x % Q;
    const long long d0 = (long long)blockIdx.x * (kThreads / Q) + threadIdx.x / Q;
    const bool live = d0 < a.D;
    const int d = live ? (int)d0 : 0, grp = d / a.Dg;
    for (int b = blockIdx.y; b < a.B; b += gridDim.y) {
        const int slot = a.slots ? a.slots[b] : b;
        E *y = (E *)a.y + b * a.sy + d;
        if (slot < 0 || slot >= a.S) {
            if (live && q == 0)
                *y = (E)0.0f;
            continue;
        }
        const float x = (float)((const E *)a.x)[b * a.sx + d];
        float v = (float)((const E *)a.dt)[b * a.sdt + d] + (a.dt_bias ? a.dt_bias[d] : 0.0f);
        const float delta = a.softplus ? softplus(v) : v, dx = delta * x;
        const E *Bm = (const E *)a.Bm + b * a.sB + (long long)grp * a.N;
        const E *Cm = (const E *)a.Cm + b * a.sC + (long long)grp * a.N;
        const float *A = a.A + (long long)d * a.N;
        float *st = a.state + ((long long)slot * a.D + d) * a.N;
        float sum = 0.0f;
        for (int n0 = 4 * q; n0 < a.N; n0 += 4 * Q) {
            const int left = a.N - n0;
            float h[4], av[4], bv[4], cv[4];
            load_upto<float, 4>(st + n0, left, h);
            load_upto<float, 4>(A + n0, left, av);
            load_upto<E, 4>(Bm + n0, left, bv);
            load_upto<E, 4>(Cm + n0, left, cv);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                h[i] = __builtin_fmaf(__builtin_amdgcn_exp2f(av[i] * kLog2e * delta), h[i],
                                      dx * bv[i]);
                if (i < left)
                    sum = __builtin_fmaf(cv[i], h[i], sum);
            }
            if (live)
                store_upto<float, 4>(st + n0, left, h);
        }
#pragma unroll
        for (int m = 1; m < Q; m <<= 1)
            sum += __shfl_xor(sum, m, 64);
        if (live && q == 0) {
            sum = __builtin_fmaf(a.Dskip ? a.Dskip[d] : 0.0f, x, sum);
            if (a.z)
                sum *= silu((float)((const E *)a.z)[b * a.sz + d]);
            *y = (E)sum;
        }
    }
}

// ---- host --------------------------------------------------------------------------

constexpr int kLds = 160 * 1024;

inline bool scan_shape(int type, int B, int D, int L, int N, int G) {
    return type_size(type) && B >= 0 && D >= 1 && L >= 0 && L < (1 << 30) && N >= 1 &&
           N <= FINC_MAX_STATE && G >= 1 && D % G == 0 && (long long)B * D < (1ll << 31) - 256;
}

// Positions a lane: the gradients' parts and the states' layout depend on it.
// More than 32 states need 16 waves in the gradients, whose registers hold four.
inline int lane_positions(int L, int N) { return L <= 64 || N > 32 ? 4 : 8; }
inline long long part_count(int L, int N) {
    return cdivll(L > 0 ? L : 1, 16 * lane_positions(L, N));
}

inline size_t forward_lds(int N, int T, int W) {
    return ((size_t)2 * N * 16 * T + 2 * (16 / W) * N + (W > 1 ? 4 * 64 * T : 0)) * 4;
}

template <typename E, int T, int W>
int launch_forward(ScanArgs &c, hipStream_t s) {
    c.blocks = (int)cdivll(c.Dg, 16 / W);
    const long long grid = (long long)c.blocks * c.G * c.B;
    const size_t lds = forward_lds(c.N, T, W);
    if (grid >= (1ll << 31) || lds > (size_t)kLds)
        return FINC_EUNSUPPORTED;
    if (lds > 64 * 1024)
        (void)hipFuncSetAttribute((const void *)scan_forward_kernel<E, T, W>,
                                  hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    (void)hipGetLastError();   // the launch check decides
    hipLaunchKernelGGL((scan_forward_kernel<E, T, W>), dim3((unsigned)grid), dim3(kThreads),
                       (unsigned)lds, s, c);
    return launched();
}

// The parts of the arguments that both directions check and use.
bool scan_common(const finc_scan_args *a, ScanArgs &c) {
    c = ScanArgs{};
    c.x = rows_of(a->x);
    c.dt = rows_of(a->dt);
    c.z = rows_of(a->z);
    c.Bm = rows_of(a->Bm);
    c.Cm = rows_of(a->Cm);
    c.A = a->A;
    c.Dskip = a->Dskip;
    c.dt_bias = a->dt_bias;
    c.lengths = a->lengths;
    c.states = a->states;
    c.B = a->B;
    c.D = a->D;
    c.L = a->L;
    c.N = a->N;
    c.G = a->G;
    c.Dg = a->D / a->G;
    c.softplus = a->softplus;
    c.parts = (int)part_count(a->L, a->N);
    return true;
}

// The gradients' waves: W share the states (four each), H fours of channels.
inline int state_waves(int N) { return N <= 4 ? 1 : N <= 8 ? 2 : N <= 16 ? 4 : N <= 32 ? 8 : 16; }
inline int channel_fours(int W) { return W >= 8 ? 1 : 8 / W; }

// Channels of a set: a workgroup a compute unit where there are that many channels,
// and at most 64, which the state in LDS holds.
inline int set_channels(int B, int D, int N, int G) {
    const int step = 4 * channel_fours(state_waves(N));
    long long c = cdivll(cdivll((long long)B * D, 256), step) * step;
    const long long most = cdivll(D / G, step) * step;
    c = c < most ? c : most;
    return (int)(c < step ? step : c > 64 ? 64 : c);
}

template <typename E, int T, int W, int H>
int launch_backward(GradArgs &c, hipStream_t s) {
    const long long grid = (long long)c.sets * c.f.G * c.f.B;
    const size_t lds = backward_lds(c.f.N, T, W, H, c.set);
    if (grid >= (1ll << 31) || lds > (size_t)kLds)
        return FINC_EUNSUPPORTED;
    if (lds > 64 * 1024)
        (void)hipFuncSetAttribute((const void *)scan_backward_kernel<E, T, W, H>,
                                  hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    (void)hipGetLastError();   // the launch check decides
    hipLaunchKernelGGL((scan_backward_kernel<E, T, W, H>), dim3((unsigned)grid),
                       dim3(64 * W * H), (unsigned)lds, s, c);
    return launched();
}

template <typename E>
int dispatch_backward(GradArgs &c, hipStream_t s) {
    const int W = state_waves(c.f.N);
    if (W == 16)
        return launch_backward<E, 4, 16, 1>(c, s);
    if (lane_positions(c.f.L, c.f.N) == 4)
        return W == 1   ? launch_backward<E, 4, 1, 8>(c, s)
               : W == 2 ? launch_backward<E, 4, 2, 4>(c, s)
               : W == 4 ? launch_backward<E, 4, 4, 2>(c, s)
                        : launch_backward<E, 4, 8, 1>(c, s);
    return W == 1   ? launch_backward<E, 8, 1, 8>(c, s)
           : W == 2 ? launch_backward<E, 8, 2, 4>(c, s)
           : W == 4 ? launch_backward<E, 8, 4, 2>(c, s)
                    : launch_backward<E, 8, 8, 1>(c, s);
}

inline size_t up256(size_t n) { return (n + 255) / 256 * 256; }
inline size_t shared_bytes(int B, int D, int L, int N, int G) {
    return up256((size_t)2 * cdivll(D / G, set_channels(B, D, N, G)) * B * G * N * L * 4);
}

}  // namespace

extern "C" {

size_t finc_selective_scan_states_bytes(int B, int D, int L, int N) {
    if (!scan_shape(FINC_F32, B, D, L, N, 1))
        return 0;
    return ((size_t)B * D * part_count(L, N) * N * 4 + 255) / 256 * 256;
}

int finc_selective_scan_forward(const finc_scan_args *a, hipStream_t stream) {
    if (!a || !scan_shape(a->type, a->B, a->D, a->L, a->N, a->G) || ((uintptr_t)a->states & 255u))
        return FINC_EINVAL;
    const int sz = type_size(a->type), B = a->B, D = a->D, L = a->L;
    const long long st = (long long)B * D * a->N, GN = (long long)a->G * a->N;
    const Region in[] = {raster(a->x, B, D, L, sz), raster(a->dt, B, D, L, sz),
                         a->z.p ? raster(a->z, B, D, L, sz) : flat(nullptr, 0, sz),
                         raster(a->Bm, B, (int)GN, L, sz), raster(a->Cm, B, (int)GN, L, sz),
                         flat(a->A, (long long)D * a->N, 4), flat(a->Dskip, a->Dskip ? D : 0, 4),
                         flat(a->dt_bias, a->dt_bias ? D : 0, 4),
                         flat(a->lengths, a->lengths ? B : 0, 4),
                         flat(a->state != a->state_out ? a->state : nullptr,
                              a->state && a->state != a->state_out ? st : 0, 4)};
    const Region out[] = {
        raster(a->y, B, D, L, sz), flat(a->state_out, a->state_out ? st : 0, 4),
        flat(a->states,
             a->states ? (long long)finc_selective_scan_states_bytes(B, D, L, a->N) / 4 : 0, 4)};
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
    ScanArgs c;
    scan_common(a, c);
    c.y = rows_of(a->y);
    c.state = a->state;
    c.state_out = a->state_out;
    int rc = FINC_EINVAL;
    // 2048 waves are two a SIMD
    const bool few = (long long)B * D < 4 * 2048;
    with_type(a->type, [&](auto e) {
        typedef decltype(e) E;
        if (lane_positions(L, a->N) == 4)
            rc = few ? launch_forward<E, 4, 4>(c, stream) : launch_forward<E, 4, 1>(c, stream);
        else
            rc = few ? launch_forward<E, 8, 4>(c, stream) : launch_forward<E, 8, 1>(c, stream);
    });
    return rc;
}

size_t finc_selective_scan_workspace_bytes(int B, int D, int L, int N, int G) {
    if (!scan_shape(FINC_F32, B, D, L, N, G))
        return 0;
    return shared_bytes(B, D, L, N, G) + up256((size_t)B * D * (N + 2) * 4);
}

int finc_selective_scan_backward(const finc_scan_args *a, const finc_scan_grads *g,
                                 hipStream_t stream) {
    if (!a || !g || !scan_shape(a->type, a->B, a->D, a->L, a->N, a->G) || !g->dA ||
        ((uintptr_t)a->states & 255u) || ((uintptr_t)g->workspace & 255u))
        return FINC_EINVAL;
    const int sz = type_size(a->type), B = a->B, D = a->D, L = a->L, N = a->N, G = a->G;
    const long long st = (long long)B * D * N;
    const int GN = G * N;
    const Region none = flat(nullptr, 0, 4);
    const Region in[] = {
        raster(a->x, B, D, L, sz), raster(a->dt, B, D, L, sz),
        a->z.p ? raster(a->z, B, D, L, sz) : none, raster(a->Bm, B, GN, L, sz),
        raster(a->Cm, B, GN, L, sz), raster(g->dy, B, D, L, sz),
        flat(a->A, (long long)D * N, 4), flat(a->Dskip, a->Dskip ? D : 0, 4),
        flat(a->dt_bias, a->dt_bias ? D : 0, 4), flat(a->lengths, a->lengths ? B : 0, 4),
        flat(g->dstate_out, g->dstate_out ? st : 0, 4),
        flat(a->states, (long long)finc_selective_scan_states_bytes(B, D, L, N) / 4, 4)};
    const Region out[] = {
        raster(g->dx, B, D, L, sz), raster(g->ddt, B, D, L, sz),
        a->z.p ? raster(g->dz, B, D, L, sz) : none, raster(g->dBm, B, GN, L, sz),
        raster(g->dCm, B, GN, L, sz), flat(g->dA, (long long)D * N, 4),
        flat(g->dDskip, g->dDskip ? D : 0, 4), flat(g->ddt_bias, g->ddt_bias ? D : 0, 4),
        flat(g->dstate, g->dstate ? st : 0, 4),
        flat(g->workspace, (long long)finc_selective_scan_workspace_bytes(B, D, L, N, G), 1)};
    for (const Region &r : in)
        if (!readable(r))
            return FINC_EINVAL;
    for (const Region &r : out)
        if (!writable(r))
            return FINC_EINVAL;
    if (!disjoint(in, out))
        return FINC_EINVAL;
    GradArgs c = {};
    scan_common(a, c.f);
    c.dy = rows_of(g->dy);
    c.dx = rows_of(g->dx);
    c.ddt = rows_of(g->ddt);
    c.dz = rows_of(g->dz);
    c.dstate_out = g->dstate_out;
    c.dstate = g->dstate;
    c.shared = (float *)g->workspace;
    c.params = (float *)((char *)g->workspace + shared_bytes(B, D, L, N, G));
    c.set = set_channels(B, D, N, G);
    c.sets = (int)cdivll(c.f.Dg, c.set);
    int rc = FINC_OK;
    const long long sums = 2ll * B * GN * cdivll(L, 1024);
    if (sums >= (1ll << 31))
        return FINC_EUNSUPPORTED;
    if (B > 0) {
        with_type(a->type, [&](auto e) { rc = dispatch_backward<decltype(e)>(c, stream); });
        if (rc != FINC_OK)
            return rc;
    }
    if (sums > 0) {
        with_type(a->type, [&](auto e) {
            hipLaunchKernelGGL(shared_sum_kernel<decltype(e)>, dim3((unsigned)sums), dim3(256), 0,
                               stream, c, rows_of(g->dBm), rows_of(g->dCm));
        });
        rc = launched();
        if (rc != FINC_OK)
            return rc;
    }
    hipLaunchKernelGGL(param_sum_kernel, dim3((unsigned)cdivll((long long)D * (N + 2), 32)),
                       dim3(256), 0, stream, c, g->dA, g->dDskip, g->ddt_bias);
    return launched();
}

int finc_selective_scan_step(const finc_scan_step_args *a, hipStream_t stream) {
    if (!a || !scan_shape(a->type, a->B, a->D, 1, a->N, a->G) || a->S < 0 ||
        (!a->slots && a->S < a->B))
        return FINC_EINVAL;
    const int sz = type_size(a->type), B = a->B, D = a->D;
    const long long GN = (long long)a->G * a->N;
    const Region in[] = {{a->x, B, a->sx, 1, 0, D, sz}, {a->dt, B, a->sdt, 1, 0, D, sz},
                         {a->z, a->z ? B : 0, a->sz, 1, 0, D, sz},
                         {a->Bm, B, a->sB, 1, 0, GN, sz}, {a->Cm, B, a->sC, 1, 0, GN, sz},
                         flat(a->A, (long long)D * a->N, 4), flat(a->Dskip, a->Dskip ? D : 0, 4),
                         flat(a->dt_bias, a->dt_bias ? D : 0, 4),
                         flat(a->slots, a->slots ? B : 0, 4)};
    const Region out[] = {{a->y, B, a->sy, 1, 0, D, sz},
                          flat(a->state, (long long)a->S * D * a->N, 4)};
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
    const StepArgs c = {a->x, a->dt, a->z, a->Bm, a->Cm, a->y, a->A, a->Dskip, a->dt_bias,
                        a->state, a->slots, a->sx, a->sdt, a->sz, a->sB, a->sC, a->sy,
                        B, a->S, D, a->N, a->G, D / a->G, a->softplus};
    with_type(a->type, [&](auto e) {
        typedef decltype(e) E;
        const unsigned gy = (unsigned)(B < 32768 ? B : 32768);
        if (a->N <= 4)
            hipLaunchKernelGGL((scan_step_kernel<E, 1>), dim3((unsigned)cdivll(D, kThreads), gy),
                               dim3(kThreads), 0, stream, c);
        else
            hipLaunchKernelGGL((scan_step_kernel<E, 4>),
                               dim3((unsigned)cdivll(D, kThreads / 4), gy), dim3(kThreads), 0,
                               stream, c);
    });
    return launched();
}

}  // extern "C"
