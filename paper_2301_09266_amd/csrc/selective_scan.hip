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
    int softplus, parts;     // parts: that states are kept for, of the whole raster
    int every;               // a forward's lanes between two of them
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

// S states of a row's part: adds C h to y, and gives the states at the start of the
// lane's run and at the part's end (in the row's last lane); `in` are the states
// before the part.
template <int T, int S>
__device__ inline void scan_states(const float *tb, const float *tc, const int (&n)[S],
                                   const float (&A2)[S], const float (&in)[S], int lane,
                                   const float (&delta)[T], const float (&dx)[T], float sum,
                                   float (&y)[T], float (&start)[S], float (&end)[S]) {
    float a[S][T], b[S][T], m[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        end[s] = 0.0f;
#pragma unroll
        for (int j4 = 0; j4 < T / 4; ++j4) {
            const float4 v = *(const float4 *)(tb + tile_at<T>(n[s], j4, lane));
            const float bv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = 4 * j4 + i;
                a[s][j] = __builtin_amdgcn_exp2f(A2[s] * delta[j]);
                b[s][j] = dx[j] * bv[i];
                end[s] = j ? __builtin_fmaf(a[s][j], end[s], b[s][j]) : b[s][j];
            }
        }
        m[s] = __builtin_amdgcn_exp2f(A2[s] * sum);
    }
    scan_up(m, end);
#pragma unroll
    for (int s = 0; s < S; ++s) {
        end[s] = __builtin_fmaf(m[s], in[s], end[s]);
        float h = start[s] = neighbour<kFromLower>(in[s], end[s]);
#pragma unroll
        for (int j4 = 0; j4 < T / 4; ++j4) {
            const float4 v = *(const float4 *)(tc + tile_at<T>(n[s], j4, lane));
            const float cv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = 4 * j4 + i;
                h = __builtin_fmaf(a[s][j], h, b[s][j]);
                y[j] = __builtin_fmaf(cv[i], h, y[j]);
            }
        }
    }
}

// Position t of a part in its channel's or its state's slots (see tile_at).
template <int T>
__device__ inline int slot_at(int t) {
    return ((t % T / 4) * 16 + t / T) * 4 + t % 4;
}

// Elements as they lie in memory, for loads that are under way while others are used;
// 0 past `count`.
template <typename E, int N>
__device__ inline typename Vec<E, N>::type load_raw(const E *p, int count) {
    typename Vec<E, N>::type v;
    if (count >= N)
        return *(const typename Vec<E, N>::type *)p;
#pragma unroll
    for (int i = 0; i < N; ++i)
        v[i] = (E)0.0f;
    if (count > 0) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = p[min(i, count - 1)];
#pragma unroll
        for (int i = 1; i < N; ++i)
            v[i] = i < count ? v[i] : (E)0.0f;
    }
    return v;
}

constexpr int kUnit = 8;   // elements of B and C that a thread moves at once

// What a thread loads of B and C for one part: unit u of 2 N P / 8.
template <typename E, int T>
__device__ inline typename Vec<E, kUnit>::type load_tile(const ScanArgs &a, int b, int grp, int u,
                                                         int p0, int n_pos) {
    constexpr int Q = 16 * T / kUnit;
    const int r = u / Q, q = (u % Q) * kUnit;
    const E *row = (r >= a.N ? a.Cm : a.Bm)
                       .row<const E>(b, (long long)grp * a.N + (r >= a.N ? r - a.N : r));
    return load_raw<E, kUnit>(row + p0 + q, n_pos - p0 - q);
}
template <typename E, int T>
__device__ inline void store_tile(float *tb, int u, typename Vec<E, kUnit>::type v) {
    constexpr int Q = 16 * T / kUnit;
    const int r = u / Q, q = (u % Q) * kUnit;   // C's rows follow B's
#pragma unroll
    for (int k = 0; k < kUnit; k += 4)
        *(float4 *)(tb + r * 16 * T + slot_at<T>(q + k)) =
            make_float4((float)v[k], (float)v[k + 1], (float)v[k + 2], (float)v[k + 3]);
}

// One block: CB = 16 / W channels of one batch row and group.  W waves share a
// channel's states (each N / W of them) where there are few channels; then a wave
// prepares one channel's positions for all of them and sums that channel's outputs.
// The next part's loads are under way while a part is computed.
template <typename E, int T, int W>
__global__ __launch_bounds__(kThreads, 2) void scan_forward_kernel(ScanArgs a) {
    constexpr int CB = 16 / W, P = 16 * T;   // P: positions of a part
    constexpr int I = T / W;                 // positions that a thread prepares
    constexpr int K = 4;                     // units of B and C loaded ahead
    extern __shared__ __attribute__((aligned(16))) float lds[];
    float *tb = lds, *tc = tb + a.N * P;
    float *hs = tc + a.N * P;                // the states between parts, CB x N
    float *As = hs + CB * a.N;               // A log2 e, CB x N
    float *pre = As + CB * a.N;              // W > 1: delta, delta x of CB channels
    float *red = pre + 2 * CB * P;           // W > 1: the waves' sums of y
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 15, rowi = (tid >> 4) & 3;
    int blk = blockIdx.x;
    const int cb = blk % a.blocks;
    blk /= a.blocks;
    const int grp = blk % a.G, b = blk / a.G;
    const int split = wave % W;
    const int cl = W > 1 ? rowi : wave * 4 + rowi;   // the channel whose states it scans
    const int cp = tid * I / P, pos = tid * I % P;   // the one whose positions it prepares
    const bool live = cb * CB + cp < a.Dg;
    const int d = grp * a.Dg + (live ? cb * CB + cp : 0);
    const int n_pos = row_length(a.lengths, b, a.L);
    const int units = 2 * a.N * (P / kUnit);
    for (int i = tid; i < CB * a.N; i += kThreads) {
        const int c = i / a.N, n = i - c * a.N, dd = cb * CB + c;
        const bool ok = dd < a.Dg;
        const long long at = (long long)(grp * a.Dg + (ok ? dd : 0)) * a.N + n;
        As[i] = ok ? a.A[at] * kLog2e : 0.0f;
        hs[i] = ok && a.state ? a.state[(long long)b * a.D * a.N + at] : 0.0f;
    }
    const float bias = a.dt_bias ? a.dt_bias[d] : 0.0f;
    const float skip = a.Dskip ? a.Dskip[d] : 0.0f;
    const E *xr = a.x.row<const E>(b, d) + pos, *dr = a.dt.row<const E>(b, d) + pos;
    const E *zr = a.z.p ? a.z.row<const E>(b, d) + pos : nullptr;
    E *yr = a.y.row<E>(b, d) + pos;
    const int own = live ? n_pos - pos : 0;
    const int parts = (n_pos + P - 1) / P;
    typename Vec<E, I>::type nx, nd, nz;
    typename Vec<E, kUnit>::type nt[K];
    if (parts > 0) {
        nx = load_raw<E, I>(xr, own);
        nd = load_raw<E, I>(dr, own);
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (tid + k * kThreads < units)
                nt[k] = load_tile<E, T>(a, b, grp, tid + k * kThreads, 0, n_pos);
    }
    for (int part = 0; part < parts; ++part) {
        const int p0 = part * P;
        // positions past the row's length: delta 0 keeps the state, B and C are 0
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (tid + k * kThreads < units)
                store_tile<E, T>(tb, tid + k * kThreads, nt[k]);
        for (int u = tid + K * kThreads; u < units; u += kThreads)
            store_tile<E, T>(tb, u, load_tile<E, T>(a, b, grp, u, p0, n_pos));
        float x[I], delta[T], dx[T], y[T];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            x[i] = (float)nx[i];
            float v = (float)nd[i] + bias;
            if (a.softplus)
                v = softplus(v);
            delta[i] = keep_if(i < own - p0, v);
            dx[i] = delta[i] * x[i];
        }
        if (W > 1) {
            float *q = pre + cp * P + slot_at<T>(pos);
#pragma unroll
            for (int i = 0; i < I; ++i) {
                q[i] = delta[i];
                q[CB * P + i] = dx[i];
            }
        }
        __syncthreads();
        // under way until the part is done
        if (zr)
            nz = load_raw<E, I>(zr + p0, own - p0);
        if (part + 1 < parts) {
            nx = load_raw<E, I>(xr + p0 + P, own - p0 - P);
            nd = load_raw<E, I>(dr + p0 + P, own - p0 - P);
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (tid + k * kThreads < units)
                    nt[k] = load_tile<E, T>(a, b, grp, tid + k * kThreads, p0 + P, n_pos);
        }
        float sum = 0.0f;
#pragma unroll
        for (int j4 = 0; j4 < T / 4; ++j4) {
            if (W > 1) {
                const float *q = pre + cl * P + (j4 * 16 + lane) * 4;
                const float4 u = *(const float4 *)q, v = *(const float4 *)(q + CB * P);
                delta[4 * j4] = u.x;
                delta[4 * j4 + 1] = u.y;
                delta[4 * j4 + 2] = u.z;
                delta[4 * j4 + 3] = u.w;
                dx[4 * j4] = v.x;
                dx[4 * j4 + 1] = v.y;
                dx[4 * j4 + 2] = v.z;
                dx[4 * j4 + 3] = v.w;
            }
#pragma unroll
            for (int j = 4 * j4; j < 4 * j4 + 4; ++j) {
                sum += delta[j];
                y[j] = 0.0f;
            }
        }
        const int cs = cb * CB + cl;
        // states are kept every a.every lanes' runs, for the gradients
        float *kept = a.states && cs < a.Dg && lane % a.every == 0
                          ? a.states + ((((long long)b * a.D + grp * a.Dg + cs) * a.parts +
                                         (long long)part * (16 / a.every) + lane / a.every) *
                                        a.N)
                          : nullptr;
        if (kept && p0 + lane * T >= n_pos)
            kept = nullptr;   // its part is not in the row
        float *hr = hs + cl * a.N;
        const float *Ar = As + cl * a.N;
        int i = split;
        for (; i + W < a.N; i += 2 * W) {
            const int n[2] = {i, i + W};
            const float A2[2] = {Ar[n[0]], Ar[n[1]]}, in[2] = {hr[n[0]], hr[n[1]]};
            float start[2], end[2];
            scan_states<T, 2>(tb, tc, n, A2, in, lane, delta, dx, sum, y, start, end);
            if (kept) {
                kept[n[0]] = start[0];
                kept[n[1]] = start[1];
            }
            if (lane == 15) {
                hr[n[0]] = end[0];
                hr[n[1]] = end[1];
            }
        }
        for (; i < a.N; i += W) {
            const int n[1] = {i};
            const float A2[1] = {Ar[i]}, in[1] = {hr[i]};
            float start[1], end[1];
            scan_states<T, 1>(tb, tc, n, A2, in, lane, delta, dx, sum, y, start, end);
            if (kept)
                kept[i] = start[0];
            if (lane == 15)
                hr[i] = end[0];
        }
        if (W > 1) {
            float4 *r = (float4 *)red + (wave * (T / 4)) * 64 + (tid & 63);
#pragma unroll
            for (int j4 = 0; j4 < T / 4; ++j4)
                r[j4 * 64] = make_float4(y[4 * j4], y[4 * j4 + 1], y[4 * j4 + 2], y[4 * j4 + 3]);
            __syncthreads();
            const float *q = red + cp * 64 + slot_at<T>(pos) % 64 + slot_at<T>(pos) / 64 * 256;
#pragma unroll
            for (int i = 0; i < I; ++i) {
                y[i] = q[i];
#pragma unroll
                for (int w = 1; w < W; ++w)
                    y[i] += q[w * (T / 4) * 256 + i];
            }
        }
        if (live) {
#pragma unroll
            for (int i = 0; i < I; ++i) {
                float v = __builtin_fmaf(skip, x[i], y[i]);
                if (zr)
                    v *= silu((float)nz[i]);
                y[i] = keep_if(i < own - p0, v);
            }
            store_upto<E, I>(yr + p0, a.L - p0 - pos, y);
        }
        // the next part's tile, and its positions, take the place of this one's
        if (W == 1)
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
// row and walks the parts from the last to the first.  A wave takes a channel at a
// time: its four rows of 16 lanes hold a quarter of the states each, S a lane, over
// the same positions.  So a lane keeps the gradients of B and C of its own states and
// positions in registers while the wave's channels pass, the sums over the states are
// sums over the four rows, and the waves meet only where a part ends.  Each row
// prepares a quarter of the positions and hands them to the others through LDS; the
// sums come back to the row that prepared them.  The states inside a part are
// recomputed from the one that the forward kept at its start.

struct GradArgs {
    ScanArgs f;
    Rows dy, dx, ddt, dz;
    const float *dstate_out;
    float *dstate;
    float *shared;    // dB then dC by sets, (2, sets, B, G N, L)
    float *params;    // dA, dDskip, ddt_bias by batch rows, (B, D (N + 2))
    int set, sets;    // channels of a set, sets of a group
};

constexpr int kGradWaves = 8;

// States a lane whose gradients the waves exchange at once.
template <int T>
constexpr int kSwap = 32 / T;

inline size_t backward_lds(int N, int T, int set) {
    return ((size_t)2 * N * 16 * T + kGradWaves * 3 * 16 * T + (size_t)3 * set * N +
            (size_t)2 * set + (size_t)2 * 32 * 64 * (kGradWaves / 2)) * 4;
}

// The sums over the four rows of T values a lane: row r gets those of positions
// r T / 4 and on.
__device__ inline float swap32(float a, float b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a),
                                                    __builtin_bit_cast(unsigned, b), false, false);
    return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
__device__ inline float swap16(float a, float b) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a),
                                                    __builtin_bit_cast(unsigned, b), false, false);
    return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
template <int T>
__device__ inline void sum_rows(const float (&v)[T], float (&out)[T / 4]) {
    float u[T / 2];
#pragma unroll
    for (int j = 0; j < T / 2; ++j)
        u[j] = swap32(v[j], v[j + T / 2]);
#pragma unroll
    for (int j = 0; j < T / 4; ++j)
        out[j] = swap16(u[j], u[j + T / 4]);
}

template <typename E, int T, int S>
__global__ __launch_bounds__(64 * kGradWaves) void scan_backward_kernel(GradArgs ga) {
    constexpr int P = 16 * T, I = T / 4, TH = 64 * kGradWaves, SW = S < kSwap<T> ? S : kSwap<T>;
    const ScanArgs &a = ga.f;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    float *tb = lds, *tc = tb + a.N * P;
    float *pre = tc + a.N * P;                     // delta, delta x, dy of a wave's channel
    float *swp = pre + kGradWaves * 3 * P;         // half the waves' gradients of B and C
    float *carry = swp + 2 * 32 * 64 * (kGradWaves / 2);   // G at the part's end, set x N
    float *As = carry + ga.set * a.N;              // A log2 e
    float *dAs = As + ga.set * a.N;                // dA
    float *ps = dAs + ga.set * a.N;                // dDskip, ddt_bias: set x 2
    const int tid = threadIdx.x, lane = tid & 15, rowi = (tid >> 4) & 3;
    // uniform: a wave's rows of activations have their addresses in scalar registers
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n0 = rowi * S;
    int blk = blockIdx.x;
    const int set = blk % ga.sets;
    blk /= ga.sets;
    const int grp = blk % a.G, b = blk / a.G;
    const int c0 = set * ga.set;                   // the set's first channel in the group
    const int count = min(ga.set, a.Dg - c0);
    const long long first = (long long)grp * a.Dg + c0;
    const int n_pos = row_length(a.lengths, b, a.L);
    const int parts = (n_pos + P - 1) / P;
    const int units = 2 * a.N * (P / kUnit);
    for (int i = tid; i < ga.set * a.N; i += TH) {
        const bool ok = i < count * a.N;
        As[i] = ok ? a.A[first * a.N + i] * kLog2e : 0.0f;
        carry[i] = ok && ga.dstate_out ? ga.dstate_out[((long long)b * a.D + first) * a.N + i] : 0.0f;
        dAs[i] = 0.0f;
    }
    for (int i = tid; i < count * 2; i += TH)
        ps[i] = 0.0f;
    // the positions of a part that this lane prepares, and the wave's place for them
    const int pos = lane * T + rowi * I;
    float *mine = pre + wave * 3 * P;
    typedef typename Vec<E, I>::type Raw;
    Raw nx, nd, ng, nz;
    float nin[S];
    auto fetch = [&](int c, int part) {
        const int d = (int)first + c, p0 = part * P, left = n_pos - p0 - pos;
        nx = load_raw<E, I>(a.x.row<const E>(b, d) + p0 + pos, left);
        nd = load_raw<E, I>(a.dt.row<const E>(b, d) + p0 + pos, left);
        ng = load_raw<E, I>(ga.dy.row<const E>(b, d) + p0 + pos, left);
        if (a.z.p)
            nz = load_raw<E, I>(a.z.row<const E>(b, d) + p0 + pos, left);
        const float *st = a.states + (((long long)b * a.D + d) * a.parts + part) * a.N;
#pragma unroll
        for (int s = 0; s < S; ++s)
            nin[s] = n0 + s < a.N ? st[n0 + s] : 0.0f;
    };
    if (parts > 0 && wave < count)
        fetch(wave, parts - 1);
    for (int part = parts - 1; part >= 0; --part) {
        const int p0 = part * P;
        for (int u = tid; u < units; u += TH)
            store_tile<E, T>(tb, u, load_tile<E, T>(a, b, grp, u, p0, n_pos));
        __syncthreads();
        float dB[S][T], dC[S][T];
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int j = 0; j < T; ++j)
                dB[s][j] = dC[s][j] = 0.0f;
        for (int c = wave; c < count; c += kGradWaves) {
            const int d = (int)first + c, left = n_pos - p0 - pos;
            float x[I], delta[I], slope[I], z[I], dout[I], dy[I], in[S];
            const float bias = a.dt_bias ? a.dt_bias[d] : 0.0f;
            const float skip = a.Dskip ? a.Dskip[d] : 0.0f;
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const float v = (float)nd[i] + bias;
                x[i] = (float)nx[i];
                dout[i] = (float)ng[i];
                slope[i] = a.softplus ? sigmoid(v) : 1.0f;
                delta[i] = keep_if(i < left, a.softplus ? softplus(v) : v);
                z[i] = a.z.p ? (float)nz[i] : 0.0f;
                dy[i] = a.z.p ? dout[i] * silu(z[i]) : dout[i];
                float *q = mine + slot_at<T>(pos + i);
                q[0] = delta[i];
                q[P] = delta[i] * x[i];
                q[2 * P] = dy[i];
            }
#pragma unroll
            for (int s = 0; s < S; ++s)
                in[s] = nin[s];
            // the next channel's, under way
            if (c + kGradWaves < count)
                fetch(c + kGradWaves, part);
            else if (part > 0)
                fetch(wave, part - 1);
            __builtin_amdgcn_wave_barrier();
            float de[T], dx[T], g[T], gB[T], sA[T], yv[T], sum = 0.0f;
#pragma unroll
            for (int j4 = 0; j4 < T / 4; ++j4) {
                const float *q = mine + (j4 * 16 + lane) * 4;
                const float4 u = *(const float4 *)q, v = *(const float4 *)(q + P);
                const float4 e = *(const float4 *)(q + 2 * P);
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
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const bool has = n0 + s < a.N;
                const int n = has ? n0 + s : 0;
                const float A2 = has ? As[c * a.N + n] : 0.0f;
                const float after = has ? carry[c * a.N + n] : 0.0f;
                float av[T], h[T], Bv[T], Cv[T], m[1], e[1] = {0.0f};
#pragma unroll
                for (int j4 = 0; j4 < T / 4; ++j4) {
                    const float4 u = *(const float4 *)(tb + tile_at<T>(n, j4, lane));
                    const float4 v = *(const float4 *)(tc + tile_at<T>(n, j4, lane));
                    Bv[4 * j4] = u.x;
                    Bv[4 * j4 + 1] = u.y;
                    Bv[4 * j4 + 2] = u.z;
                    Bv[4 * j4 + 3] = u.w;
                    Cv[4 * j4] = v.x;
                    Cv[4 * j4 + 1] = v.y;
                    Cv[4 * j4 + 2] = v.z;
                    Cv[4 * j4 + 3] = v.w;
                }
                if (!has) {   // a lane without this state adds nothing
#pragma unroll
                    for (int j = 0; j < T; ++j)
                        Bv[j] = Cv[j] = 0.0f;
                }
#pragma unroll
                for (int j = 0; j < T; ++j) {
                    av[j] = __builtin_amdgcn_exp2f(A2 * de[j]);
                    e[0] = __builtin_fmaf(av[j], e[0], dx[j] * Bv[j]);
                }
                const float run = m[0] = __builtin_amdgcn_exp2f(A2 * sum);
                scan_up(m, e);
                const float start =
                    neighbour<kFromLower>(in[s], __builtin_fmaf(m[0], in[s], e[0]));
                float prev = start;
#pragma unroll
                for (int j = 0; j < T; ++j)
                    prev = h[j] = __builtin_fmaf(av[j], prev, dx[j] * Bv[j]);
                // G below the lane's run, from 0 above it, then from the lanes above
                e[0] = 0.0f;
#pragma unroll
                for (int j = T - 1; j >= 0; --j)
                    e[0] = av[j] * __builtin_fmaf(Cv[j], g[j], e[0]);
                m[0] = run;
                scan_down(m, e);
                const float low = __builtin_fmaf(m[0], after, e[0]);
                float G = neighbour<kFromUpper>(after, low), dA = 0.0f;
#pragma unroll
                for (int j = T - 1; j >= 0; --j) {
                    const float gt = __builtin_fmaf(Cv[j], g[j], G);
                    G = av[j] * gt;
                    dC[s][j] = __builtin_fmaf(g[j], h[j], dC[s][j]);
                    dB[s][j] = __builtin_fmaf(gt, dx[j], dB[s][j]);
                    gB[j] = __builtin_fmaf(gt, Bv[j], gB[j]);
                    yv[j] = __builtin_fmaf(Cv[j], h[j], yv[j]);
                    const float t = G * (j ? h[j ? j - 1 : 0] : start);
                    sA[j] = __builtin_fmaf(A2, t, sA[j]);
                    dA = __builtin_fmaf(de[j], t, dA);
                }
                dA = row_sum(dA);
                if (has) {
                    if (lane == 15)
                        dAs[c * a.N + n] += dA;
                    if (lane == 0)
                        carry[c * a.N + n] = low;
                }
                // one state's values at a time: sums put off to the end would keep every
                // state's h and g in registers
#pragma unroll
                for (int j = 0; j < T; ++j)
                    asm volatile("" : "+v"(dB[s][j]), "+v"(dC[s][j]), "+v"(gB[j]), "+v"(sA[j]),
                                 "+v"(yv[j]));
            }
            // the gradients of the positions that this lane prepared
            float v0[I], v1[I], v2[I], ox[I], ot[I], oz[I], sD = 0.0f, sb = 0.0f;
            sum_rows<T>(gB, v0);
            sum_rows<T>(sA, v1);
            sum_rows<T>(yv, v2);
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const bool inside = i < left;
                const float dd = __builtin_fmaf(x[i], v0[i], v1[i] * 0.693147180559945309f);
                ot[i] = keep_if(inside, dd * slope[i]);
                ox[i] = keep_if(inside, __builtin_fmaf(delta[i], v0[i], skip * dy[i]));
                const float y = __builtin_fmaf(skip, x[i], v2[i]);
                oz[i] = keep_if(inside, dout[i] * y * silu_grad(z[i], sigmoid(z[i])));
                sb += ot[i];
                sD = __builtin_fmaf(dy[i], x[i], sD);
            }
            const int room = a.L - p0 - pos;
            store_upto<E, I>(ga.dx.row<E>(b, d) + p0 + pos, room, ox);
            store_upto<E, I>(ga.ddt.row<E>(b, d) + p0 + pos, room, ot);
            if (a.z.p)
                store_upto<E, I>(ga.dz.row<E>(b, d) + p0 + pos, room, oz);
            sD = wave_sum(sD);
            sb = wave_sum(sb);
            if ((tid & 63) == 0) {
                ps[2 * c] += sD;
                ps[2 * c + 1] += sb;
            }
        }
        // dB and dC of the part: the upper half of the waves to the lower, by halves
#pragma unroll
        for (int s0 = 0; s0 < S; s0 += SW) {
#pragma unroll
            for (int half = kGradWaves / 2; half; half >>= 1) {
                float *q = swp + (wave & (half - 1)) * 2 * SW * T * 64 + (tid & 63) * 4;
                if (wave >= half && wave < 2 * half)
#pragma unroll
                    for (int k = 0; k < SW * T / 4; ++k) {
                        const int s = s0 + 4 * k / T, j = 4 * k % T;
                        *(float4 *)(q + 2 * k * 256) =
                            make_float4(dB[s][j], dB[s][j + 1], dB[s][j + 2], dB[s][j + 3]);
                        *(float4 *)(q + (2 * k + 1) * 256) =
                            make_float4(dC[s][j], dC[s][j + 1], dC[s][j + 2], dC[s][j + 3]);
                    }
                __syncthreads();
                if (wave < half)
#pragma unroll
                    for (int k = 0; k < SW * T / 4; ++k) {
                        const int s = s0 + 4 * k / T, j = 4 * k % T;
                        const float4 u = *(const float4 *)(q + 2 * k * 256);
                        const float4 v = *(const float4 *)(q + (2 * k + 1) * 256);
                        dB[s][j] += u.x;
                        dB[s][j + 1] += u.y;
                        dB[s][j + 2] += u.z;
                        dB[s][j + 3] += u.w;
                        dC[s][j] += v.x;
                        dC[s][j + 1] += v.y;
                        dC[s][j + 2] += v.z;
                        dC[s][j + 3] += v.w;
                    }
                __syncthreads();
            }
        }
        if (wave == 0) {
            const long long rows = (long long)a.G * a.N;
            const int t0 = p0 + lane * T;
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (n0 + s < a.N) {
                    const long long r =
                        ((long long)set * a.B + b) * rows + (long long)grp * a.N + n0 + s;
                    store_upto<float, T>(ga.shared + r * a.L + t0, a.L - t0, dB[s]);
                    store_upto<float, T>(ga.shared + ((long long)ga.sets * a.B * rows + r) * a.L +
                                             t0,
                                         a.L - t0, dC[s]);
                }
        }
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
        out[(long long)a.D * a.N + first + c] = ps[2 * c];
        out[(long long)a.D * (a.N + 1) + first + c] = ps[2 * c + 1];
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
// More than 16 states leave the gradients' registers room for four.
inline int lane_positions(int L, int N) { return L <= 64 || N > 16 ? 4 : 8; }
inline long long part_count(int L, int N) {
    return cdivll(L > 0 ? L : 1, 16 * lane_positions(L, N));
}

inline size_t forward_lds(int N, int T, int W) {
    return ((size_t)2 * N * 16 * T + 2 * (16 / W) * N + (W > 1 ? (2 * 4 * 16 + 4 * 64) * T : 0)) * 4;
}

template <typename E, int T, int W>
int launch_forward(ScanArgs &c, hipStream_t s) {
    c.blocks = (int)cdivll(c.Dg, 16 / W);
    c.every = lane_positions(c.L, c.N) * 16 / T;
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

// Channels of a set: a workgroup a compute unit where there are that many channels,
// and at most 64, which the state in LDS holds.
inline int set_channels(int B, int D, int G) {
    long long c = cdivll(cdivll((long long)B * D, 256), kGradWaves) * kGradWaves;
    const long long most = cdivll(D / G, kGradWaves) * kGradWaves;
    c = c < most ? c : most;
    return (int)(c > 64 ? 64 : c);
}

template <typename E, int T, int S>
int launch_backward(GradArgs &c, hipStream_t s) {
    const long long grid = (long long)c.sets * c.f.G * c.f.B;
    const size_t lds = backward_lds(c.f.N, T, c.set);
    if (grid >= (1ll << 31) || lds > (size_t)kLds)
        return FINC_EUNSUPPORTED;
    (void)hipFuncSetAttribute((const void *)scan_backward_kernel<E, T, S>,
                              hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    (void)hipGetLastError();   // the launch check decides
    hipLaunchKernelGGL((scan_backward_kernel<E, T, S>), dim3((unsigned)grid),
                       dim3(64 * kGradWaves), (unsigned)lds, s, c);
    return launched();
}

// S states a lane, a quarter of them all.
template <typename E>
int dispatch_backward(GradArgs &c, hipStream_t s) {
    const int N = c.f.N;
    if (lane_positions(c.f.L, N) == 4)
        return N <= 4    ? launch_backward<E, 4, 1>(c, s)
               : N <= 8  ? launch_backward<E, 4, 2>(c, s)
               : N <= 16 ? launch_backward<E, 4, 4>(c, s)
               : N <= 32 ? launch_backward<E, 4, 8>(c, s)
                         : launch_backward<E, 4, 16>(c, s);
    return N <= 4   ? launch_backward<E, 8, 1>(c, s)
           : N <= 8 ? launch_backward<E, 8, 2>(c, s)
                    : launch_backward<E, 8, 4>(c, s);
}

inline size_t up256(size_t n) { return (n + 255) / 256 * 256; }
inline size_t shared_bytes(int B, int D, int L, int N, int G) {
    return up256((size_t)2 * cdivll(D / G, set_channels(B, D, G)) * B * G * N * L * 4);
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
    const int T = L <= 64 ? 4 : L <= 128 || a->N > 32 ? 8 : 16;
    with_type(a->type, [&](auto e) {
        typedef decltype(e) E;
        if (few)
            rc = T == 4   ? launch_forward<E, 4, 4>(c, stream)
                 : T == 8 ? launch_forward<E, 8, 4>(c, stream)
                          : launch_forward<E, 16, 4>(c, stream);
        else
            rc = T == 4   ? launch_forward<E, 4, 1>(c, stream)
                 : T == 8 ? launch_forward<E, 8, 1>(c, stream)
                          : launch_forward<E, 16, 1>(c, stream);
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
    c.set = set_channels(B, D, G);
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
