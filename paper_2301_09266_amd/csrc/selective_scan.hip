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
// bf16 a position's 8 bytes of activations take a fifth of their time.  Rows walk the
// raster in parts of 16 T positions with the state in LDS between them.
#include "seq_common.h"

namespace {

using namespace finc_seq;

constexpr int kThreads = 512;
constexpr float kLog2e = 1.44269504088896341f;

// A log2 e, finite: an infinite decay times padding's step of 0 has no value, which the
// next state would take over.  Steps above 1e-36 still take its exponential to 0 or
// infinity.
__device__ inline float decay(float a) {
    const float v = a * kLog2e;
    return __builtin_fabsf(v) > 3e38f ? __builtin_copysignf(3e38f, v) : v;
}

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
    int NP;                  // states that are kept: N with those that fill four rows
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
// Both directions at once: (a, h) over the lanes before, (c, g) over the lanes after.
#define FINC_BOTH(n)                                                                        \
    "v_fmac_f32_dpp %1, %1, %0 row_shr:" n " row_mask:0xf bank_mask:0xf\n"                 \
    "v_fmac_f32_dpp %3, %3, %2 row_shl:" n " row_mask:0xf bank_mask:0xf\n"                 \
    "v_mul_f32_dpp %0, %0, %0 row_shr:" n " row_mask:0xf bank_mask:0xf\n"                  \
    "v_mul_f32_dpp %2, %2, %2 row_shl:" n " row_mask:0xf bank_mask:0xf\n"
__device__ inline void scan_both(float &a, float &h, float &c, float &g) {
    asm volatile("s_nop 1\n" FINC_BOTH("1") FINC_BOTH("2") FINC_BOTH("4") FINC_BOTH("8") "s_nop 1"
                 : "+v"(a), "+v"(h), "+v"(c), "+v"(g));
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

// S states of a row's part: adds C h to y, and gives the states at the part's end (in
// the row's last lane); `in` are the states before the part.
template <int T, int S>
__device__ inline void scan_states(const float *tb, const float *tc, const int (&n)[S],
                                   const float (&A2)[S], const float (&in)[S], int lane,
                                   const float (&delta)[T], const float (&dx)[T], float sum,
                                   float (&y)[T], float (&end)[S]) {
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
        float h = neighbour<kFromLower>(in[s], end[s]);
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

// S floats of LDS, aligned to their size (to 16 bytes above four).
template <int S>
__device__ inline void lds_load(const float *p, float *v) {
    constexpr int C = S < 4 ? S : 4;
    typedef float Q __attribute__((ext_vector_type(C)));
#pragma unroll
    for (int i = 0; i < S; i += C) {
        const Q q = *(const Q *)(p + i);
#pragma unroll
        for (int k = 0; k < C; ++k)
            v[i + k] = q[k];
    }
}
template <int S>
__device__ inline void lds_store(float *p, const float *v) {
    constexpr int C = S < 4 ? S : 4;
    typedef float Q __attribute__((ext_vector_type(C)));
#pragma unroll
    for (int i = 0; i < S; i += C) {
        Q q;
#pragma unroll
        for (int k = 0; k < C; ++k)
            q[k] = v[i + k];
        *(Q *)(p + i) = q;
    }
}

// Element i of a row whose address the whole wave shares: a scalar base and a 32-bit
// offset of bytes, which is formed where it is used (the sums of all rows' addresses,
// kept over a loop, would take the registers).
template <typename E>
__device__ inline E *at(E *row, unsigned i) {
    unsigned o = i * (unsigned)sizeof(E);
    asm volatile("" : "+v"(o));
    return (E *)((char *)row + o);
}
template <typename E>
__device__ inline const E *at(const E *row, unsigned i) {
    return at((E *)row, i);
}

// Elements as they lie in memory, for loads that are under way while others are used.
template <typename E, int N>
__device__ inline typename Vec<E, N>::type load_whole(const E *p) {
    return *(const typename Vec<E, N>::type *)p;
}
// The same, 0 past `count`.
template <typename E, int N>
__device__ inline typename Vec<E, N>::type load_part(const E *p, int count) {
    typename Vec<E, N>::type v;
#pragma unroll
    for (int i = 0; i < N; ++i)
        v[i] = (E)0.0f;
    if (count > 0) {
        const int n = afresh(count);
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = p[min(i, n - 1)];
#pragma unroll
        for (int i = 1; i < N; ++i)
            v[i] = i < n ? v[i] : (E)0.0f;
    }
    return v;
}
// `whole`, that every lane has all of them, is the same in the whole wave: a branch of
// some lanes would wait for the loads of the others, whose registers it fills.  For the
// same reason what is loaded ahead is loaded in every round, the last one's place again
// where nothing follows: a value that a round may leave as it was is copied, which
// waits for it.
template <typename E, int N>
__device__ inline typename Vec<E, N>::type load_raw(const E *p, int count, bool whole) {
    return whole ? load_whole<E, N>(p) : load_part<E, N>(p, count);
}

// Where N elements from `pos` of a row of L are loaded, or its last N where they would
// pass its end: bytes from the row's start.  One load in every lane, which is waited for
// only where settle() uses it.
template <typename E, int N>
__device__ inline unsigned back(int pos, int L) {
    unsigned o = (unsigned)min(pos, L - N) * (unsigned)sizeof(E);
    asm volatile("" : "+v"(o));   // formed where it is used (see at())
    return o;
}
template <typename E, int N>
__device__ inline typename Vec<E, N>::type load_back(const E *row, unsigned o) {
    return load_whole<E, N>((const E *)((const char *)row + o));
}
// Those of load_back at their places, 0 from n_pos on.
template <typename E, int N>
__device__ inline void settle(typename Vec<E, N>::type v, int pos, int L, int n_pos,
                              float (&out)[N]) {
    static_assert(N <= 2, "one element to move");
    out[N - 1] = keep_if(pos + N - 1 < n_pos, (float)v[N - 1]);
    if (N == 2)
        out[0] = keep_if(pos < n_pos, (float)(pos + N > L ? v[N - 1] : v[0]));
}
template <typename E, int N>
__device__ inline void convert(typename Vec<E, N>::type v, float (&out)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        out[i] = (float)v[i];
}

constexpr int kUnit = 8;   // elements of B and C that a thread moves at once

// What a thread loads of B and C for one part: unit u of 2 N P / 8, the row's last
// elements where the unit passes its end.  `whole`: the raster has a unit's elements.
__device__ inline int unit_at(int pos, int L) { return L < kUnit ? pos : min(pos, L - kUnit); }
template <typename E, int T>
__device__ inline typename Vec<E, kUnit>::type load_tile(const ScanArgs &a, int b, int grp, int u,
                                                         int p0, int n_pos, bool whole) {
    constexpr int Q = 16 * T / kUnit;
    const int r = u / Q, pos = p0 + (u % Q) * kUnit;
    const E *row = (r >= a.N ? a.Cm : a.Bm)
                       .row<const E>(b, (long long)grp * a.N + (r >= a.N ? r - a.N : r));
    return load_raw<E, kUnit>(row + unit_at(pos, a.L), n_pos - pos, whole);
}
template <typename E, int T>
__device__ inline void store_tile(const ScanArgs &a, float *tb, float *tc, int u, int p0, int n_pos,
                                  typename Vec<E, kUnit>::type v) {
    constexpr int Q = 16 * T / kUnit;
    const int r = u / Q;
    float *to = r >= a.N ? tc + (r - a.N) * 16 * T : tb + r * 16 * T;
    int q = (u % Q) * kUnit;
    if (p0 + 16 * T <= n_pos) {
#pragma unroll
        for (int k = 0; k < kUnit; k += 4)
            *(float4 *)(to + slot_at<T>(q + k)) =
                make_float4((float)v[k], (float)v[k + 1], (float)v[k + 2], (float)v[k + 3]);
        return;
    }
    q = afresh(q);
#pragma unroll
    for (int k = 0; k < kUnit; k += 4)
        *(float4 *)(to + slot_at<T>(q + k)) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const int first = unit_at(p0 + q, a.L) - p0;   // in the part, or before it
#pragma unroll
    for (int k = 0; k < kUnit; ++k)
        if (first + k >= q && first + k < n_pos - p0)
            to[slot_at<T>(first + k)] = (float)v[k];
}

// The forward's tiles: two in LDS, and the loads of one more; the raster exceeds a unit.
// Up to K units a thread are loaded ahead, which covers 16 states; the others are loaded as
// they are stored.
template <typename E, int T>
struct Tiles {
    static constexpr int P = 16 * T, K = 2 * 16 * P / kUnit / kThreads > 0 ? 2 * 16 * P / kUnit / kThreads : 1;
    const ScanArgs &a;
    float *lds;
    int b, grp, n_pos, units;
    typename Vec<E, kUnit>::type ahead[K];
    __device__ Tiles(const ScanArgs &a_, float *lds_, int b_, int grp_, int n_pos_)
        : a(a_), lds(lds_), b(b_), grp(grp_), n_pos(n_pos_), units(2 * a_.N * (P / kUnit)) {}
    __device__ float *of(int part) const { return lds + (part & 1) * 2 * a.N * P; }
    __device__ void fetch(int part) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            // fp32's tile leaves no registers for the unit's address (bf16: 3% more time)
            const int u = min((int)threadIdx.x + k * kThreads, units - 1);
            ahead[k] =
                load_tile<E, T>(a, b, grp, sizeof(E) == 4 ? afresh(u) : u, part * P, n_pos, true);
        }
    }
    // The part that was fetched.
    __device__ void store(int part) {
        float *tb = of(part), *tc = tb + a.N * P;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if ((int)threadIdx.x + k * kThreads < units)
                store_tile<E, T>(a, tb, tc, threadIdx.x + k * kThreads, part * P, n_pos, ahead[k]);
        for (int u = threadIdx.x + K * kThreads; u < units; u += kThreads)
            store_tile<E, T>(a, tb, tc, u, part * P, n_pos,
                             load_tile<E, T>(a, b, grp, u, part * P, n_pos, true));
    }
};

// The states at a part's start, kept for the gradients: those of one channel, by its
// wave, before it goes on from them.
__device__ inline void keep_states(const ScanArgs &a, int b, int d, int part, const float *hs,
                                   int lane64) {
    if (lane64 < a.N)
        a.states[(((long long)b * a.D + d) * a.parts + part) * a.NP + lane64] = hs[lane64];
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

// A wave for a channel: its four rows of lanes share the states (state n in row n % 4)
// over the same positions.  Each row prepares a quarter of them and hands them to the
// others through LDS; the sums over the states are sums over the rows, and come back
// to the row that prepared the position.  The block's waves share the tiles of B and
// C; the next part's tile is stored, and the one after it is under way, while a part
// is computed.  1 x 2048 x 4096 in bf16, N = 16: 63 us (bytes: 14), and of 4 rows
// 198: 393 vector instructions a channel and part of 128, 246 of them the states', which
// keep the ALU busy 77% of the time with the two waves a SIMD of one row, and throughout
// from four rows on.
template <typename E, int T>
__global__ __launch_bounds__(kThreads, 4) void scan_forward_kernel(ScanArgs a) {
    constexpr int CB = kThreads / 64, P = 16 * T, I = T / 4;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    float *hs = lds + 4 * a.N * P;           // the states between parts, CB x N
    float *As = hs + CB * a.N;               // A log2 e, CB x N
    float *pre = As + CB * a.N;              // delta, delta x of every wave's channel
    const int tid = threadIdx.x, lane = tid & 15, rowi = (tid >> 4) & 3;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int blk = block_of();
    const int cb = blk % a.blocks;
    blk /= a.blocks;
    const int grp = blk % a.G, b = blk / a.G;
    if (b >= a.B)
        return;
    const bool live = cb * CB + wave < a.Dg;
    const int d = grp * a.Dg + (live ? cb * CB + wave : 0);
    const int n_pos = __builtin_amdgcn_readfirstlane(row_length(a.lengths, b, a.L));
    for (int i = tid; i < CB * a.N; i += kThreads) {
        const int c = i / a.N, n = i - c * a.N, dd = cb * CB + c;
        const bool ok = dd < a.Dg;
        const long long at = (long long)(grp * a.Dg + (ok ? dd : 0)) * a.N + n;
        As[i] = ok ? decay(a.A[at]) : 0.0f;
        hs[i] = ok && a.state ? a.state[(long long)b * a.D * a.N + at] : 0.0f;
    }
    const float bias = a.dt_bias ? a.dt_bias[d] : 0.0f;
    const float skip = a.Dskip ? a.Dskip[d] : 0.0f;
    const int pos = lane * T + rowi * I;     // the first that this lane prepares
    float *mine = pre + wave * 2 * P;
    const int parts = (n_pos + P - 1) / P;
    typename Vec<E, I>::type nx, nd, nz;
    Tiles<E, T> tiles(a, lds, b, grp, n_pos);
    auto fetch = [&](int p0) {
        const E *xr = a.x.row<const E>(b, d), *dr = a.dt.row<const E>(b, d);
        const E *zr = a.z.p ? a.z.row<const E>(b, d) : xr;
        const unsigned o = back<E, I>(p0 + pos, a.L);
        nx = load_back<E, I>(xr, o);
        nd = load_back<E, I>(dr, o);
        nz = load_back<E, I>(zr, o);
    };
    if (parts > 0) {
        fetch(0);
        tiles.fetch(0);
        tiles.store(0);
        tiles.fetch(parts > 1);
    }
    __syncthreads();
    for (int part = 0; part < parts; ++part) {
        const int p0 = part * P, left = n_pos - p0 - pos;
        const float *tb = tiles.of(part), *tc = tb + a.N * P;
        if (part + 1 < parts)
            tiles.store(part + 1);
        float x[I], z[I], dt[I], delta[T], dx[T], y[T], sum = 0.0f;
        float *q = mine + slot_at<T>(pos);   // I neighbours of one slot
        if (p0 + P <= n_pos) {
            convert<E, I>(nx, x);
            convert<E, I>(nz, z);
            convert<E, I>(nd, dt);
        } else {
            settle<E, I>(nx, p0 + pos, a.L, n_pos, x);
            settle<E, I>(nz, p0 + pos, a.L, n_pos, z);
            settle<E, I>(nd, p0 + pos, a.L, n_pos, dt);
        }
#pragma unroll
        for (int i = 0; i < I; ++i) {
            float v = dt[i] + bias;
            if (a.softplus)
                v = softplus(v);
            v = keep_if(i < left, v);
            q[i] = v;
            q[P + i] = v * x[i];
        }
        // under way until the part is done
        fetch(part + 1 < parts ? p0 + P : p0);
        tiles.fetch(min(part + 2, parts - 1));
        wave_exchange();
#pragma unroll
        for (int j = 0; j < T; j += 4) {
            lds_load<4>(mine + (j * 4 + lane) * 4, delta + j);
            lds_load<4>(mine + P + (j * 4 + lane) * 4, dx + j);
        }
#pragma unroll
        for (int j = 0; j < T; ++j) {
            sum += delta[j];
            y[j] = 0.0f;
        }
        if (a.states && live)
            keep_states(a, b, d, part, hs + wave * a.N, tid & 63);
        wave_exchange();
        float *hr = hs + wave * a.N;
        const float *Ar = As + wave * a.N;
        int i = rowi;
        for (int k = a.N / 8; k; --k, i += 8) {
            const int n[2] = {i, i + 4};
            const float A2[2] = {Ar[i], Ar[i + 4]}, in[2] = {hr[i], hr[i + 4]};
            float end[2];
            scan_states<T, 2>(tb, tc, n, A2, in, lane, delta, dx, sum, y, end);
            if (lane == 15) {
                hr[i] = end[0];
                hr[i + 4] = end[1];
            }
        }
        for (int k = a.N % 8; k > 0; k -= 4, i += 4) {
            // a row without this state adds nothing
            const bool has = i < a.N;
            const int n[1] = {has ? i : 0};
            const float A2[1] = {has ? Ar[i] : 0.0f}, in[1] = {has ? hr[i] : 0.0f};
            float end[1], more[T], part_dx[T];
#pragma unroll
            for (int j = 0; j < T; ++j) {
                more[j] = 0.0f;
                part_dx[j] = keep_if(has, dx[j]);
            }
            scan_states<T, 1>(tb, tc, n, A2, in, lane, delta, part_dx, sum, more, end);
#pragma unroll
            for (int j = 0; j < T; ++j)
                y[j] += keep_if(has, more[j]);
            if (lane == 15 && has)
                hr[i] = end[0];
        }
        float v[I];
        sum_rows<T>(y, v);
#pragma unroll
        for (int j = 0; j < I; ++j) {
            v[j] = __builtin_fmaf(skip, x[j], v[j]);
            if (a.z.p)
                v[j] *= silu(z[j]);
            v[j] = keep_if(j < left, v[j]);
        }
        if (live) {
            E *yr = a.y.row<E>(b, d) + p0;
            if (p0 + P <= a.L)
                store_vec<E, I>(at(yr, pos), v);
            else
                store_upto<E, I>(at(yr, pos), a.L - p0 - pos, v);
        }
        // the next part's tile is there, and this one's place free
        __syncthreads();
    }
    // padding
    if (live) {
        E *r = a.y.row<E>(b, d);
        for (long long t = (long long)parts * P + (tid & 63); t < a.L; t += 64)
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

// ---- short rasters -------------------------------------------------------------------
// A scan over lanes would leave most of them past the raster's end.  Four lanes a
// channel, a quarter of the states each, go through the positions in order: each lane
// prepares every fourth four of them, which the others take from it by DPP, and adds up
// its states' share of y, which the four sum.  A position then takes, a lane, the
// exponential, 2 multiplies and 2 multiply-adds of each of its S states: 64 x 2048
// channels of 16 positions, N = 16, bf16, 15 us (their bytes 7; the scan over lanes 168).
template <int K>
__device__ inline float from_quad(float v) {   // lane K of each four
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(
                                         0, __builtin_bit_cast(int, v), K * 0x55, 0xf, 0xf, true));
}
template <int CTRL>
__device__ inline float add_quad(float v) {
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(
                                             0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

// Positions 4 K to 4 K + 3 of the 16 that the lanes prepared.
template <int S, int K, bool ALL>
__device__ inline void short_four(const float *tb, const float *tc, const float (&delta)[4],
                                  const float (&dx)[4], const float (&A2)[S], int states,
                                  float (&h)[S], bool own, float (&y)[4]) {
    // as many positions side by side as the registers hold
    constexpr int W = S <= 4 ? 4 : S == 8 ? 2 : 1;
#pragma unroll
    for (int j0 = 0; j0 < 4; j0 += W) {
        float Bv[W][S], Cv[W][S], av[W][S], v[W];
#pragma unroll
        for (int j = 0; j < W; ++j) {
            lds_load<S>(tb + (4 * K + j0 + j) * 4 * S, Bv[j]);
            lds_load<S>(tc + (4 * K + j0 + j) * 4 * S, Cv[j]);
        }
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const float de = from_quad<K>(delta[j0 + j]), u = from_quad<K>(dx[j0 + j]);
#pragma unroll
            for (int s = 0; s < S; ++s) {
                av[j][s] = __builtin_amdgcn_exp2f(A2[s] * de);
                Bv[j][s] *= u;
            }
        }
#pragma unroll
        for (int j = 0; j < W; ++j) {
            v[j] = 0.0f;
#pragma unroll
            for (int s = 0; s < S; ++s) {
                h[s] = __builtin_fmaf(av[j][s], h[s], Bv[j][s]);
                if (!ALL)
                    h[s] = keep_if(s < states, h[s]);   // 0 times an infinite input is NaN
                v[j] = __builtin_fmaf(Cv[j][s], h[s], v[j]);
            }
        }
        // over the four lanes
#pragma unroll
        for (int j = 0; j < W; ++j)
            v[j] = add_quad<0xb1>(v[j]);
#pragma unroll
        for (int j = 0; j < W; ++j) {
            v[j] = add_quad<0x4e>(v[j]);
            y[j0 + j] = own ? v[j] : y[j0 + j];
        }
    }
}

constexpr int kShortThreads = 256;

// The whole raster is one part of the gradients', at whose start the states are kept.
// ALL: N = 4 S.
template <typename E, int S, bool ALL>
__global__ __launch_bounds__(kShortThreads) void scan_short_kernel(ScanArgs a) {
    constexpr int NP = 4 * S;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const int tid = threadIdx.x, q = tid & 3, n0 = q * S, CB = blockDim.x / 4;
    int blk = block_of();
    const int cb = blk % a.blocks;
    blk /= a.blocks;
    const int grp = blk % a.G, b = blk / a.G;
    if (b >= a.B)
        return;
    const bool live = cb * CB + tid / 4 < a.Dg;
    const int d = grp * a.Dg + (live ? cb * CB + tid / 4 : 0);
    const int n_pos = __builtin_amdgcn_readfirstlane(row_length(a.lengths, b, a.L));
    const int rounds = (n_pos + 15) / 16;
    float *tb = lds, *tc = lds + rounds * 16 * NP;
    const E *xr = a.x.row<const E>(b, d) + 4 * q, *dr = a.dt.row<const E>(b, d) + 4 * q;
    const E *zr = a.z.p ? a.z.row<const E>(b, d) + 4 * q : xr;
    typename Vec<E, 4>::type nx, nd, nz;
    auto fetch = [&](int p0) {
        const int left = n_pos - p0 - 4 * q;
        const bool whole = p0 + 16 <= n_pos;
        nx = load_raw<E, 4>(xr + p0, left, whole);
        nd = load_raw<E, 4>(dr + p0, left, whole);
        nz = load_raw<E, 4>(zr + p0, left, whole);
    };
    if (rounds > 0)
        fetch(0);
    float h[S], A2[S];
    const long long at0 = ((long long)b * a.D + d) * a.N + n0;
    load_upto<float, S>(a.A + (long long)d * a.N + n0, a.N - n0, A2);
    load_upto<float, S>(a.state + at0, a.state ? a.N - n0 : 0, h);
    if (a.states && live)
        store_vec<float, S>(a.states + ((long long)b * a.D + d) * NP + n0, h);
#pragma unroll
    for (int s = 0; s < S; ++s)
        A2[s] = decay(A2[s]);
    const float bias = a.dt_bias ? a.dt_bias[d] : 0.0f;
    const float skip = a.Dskip ? a.Dskip[d] : 0.0f;
    // B and C of all positions, position by position; 0 past the raster and the states
    for (int u = tid; u < 2 * rounds * 4 * NP; u += blockDim.x) {
        const int n = u % NP, t = u / NP % (rounds * 4) * 4;
        const bool isC = u >= rounds * 4 * NP;
        const E *row = (isC ? a.Cm : a.Bm).row<const E>(b, (long long)grp * a.N + n);
        float v[4];
        load_upto<E, 4>(row + t, n < a.N ? n_pos - t : 0, v);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            (isC ? tc : tb)[(t + i) * NP + n] = v[i];
    }
    __syncthreads();
    for (int k = 0; k < rounds; ++k) {
        const int p0 = 16 * k, left = n_pos - p0 - 4 * q;
        float x[4], z[4], delta[4], dx[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = (float)nx[i];
            z[i] = (float)nz[i];
            float v = (float)nd[i] + bias;
            if (a.softplus)
                v = softplus(v);
            delta[i] = keep_if(i < left, v);
            dx[i] = delta[i] * x[i];
            y[i] = 0.0f;
            asm volatile("" : "+v"(x[i]), "+v"(z[i]));   // before the next loads
        }
        if (k + 1 < rounds)
            fetch(p0 + 16);
        const float *bp = tb + p0 * NP + n0, *cp = tc + p0 * NP + n0;
        short_four<S, 0, ALL>(bp, cp, delta, dx, A2, a.N - n0, h, q == 0, y);
        if (p0 + 4 < n_pos)
            short_four<S, 1, ALL>(bp, cp, delta, dx, A2, a.N - n0, h, q == 1, y);
        if (p0 + 8 < n_pos)
            short_four<S, 2, ALL>(bp, cp, delta, dx, A2, a.N - n0, h, q == 2, y);
        if (p0 + 12 < n_pos)
            short_four<S, 3, ALL>(bp, cp, delta, dx, A2, a.N - n0, h, q == 3, y);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[i] = __builtin_fmaf(skip, x[i], y[i]);
            if (a.z.p)
                y[i] *= silu(z[i]);
            y[i] = keep_if(i < left, y[i]);
        }
        if (live)
            store_upto<E, 4>(a.y.row<E>(b, d) + p0 + 4 * q, a.L - p0 - 4 * q, y);
    }
    if (!live)
        return;
    // padding
    const float none[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int t = rounds * 16 + 4 * q; t < a.L; t += 16)
        store_upto<E, 4>(a.y.row<E>(b, d) + t, a.L - t, none);
    if (a.state_out)
        store_upto<float, S>(a.state_out + at0, a.N - n0, h);
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
//
// Bound by the vector ALU: 894 instructions a channel and part of 128 positions at N =
// 16, 568 of them the states' (an exponential and 17 others a position), which two waves
// a SIMD, all that the gradients of B and C in registers leave, keep 80% busy.  4 x 2048 x
// 4096 in bf16 with the forward and the sums: 738 us (bytes: 155).  More than 32 states do
// not fit (43 to 47 vector registers spill), which their time does not show: 4 x 1024 x 1024
// with 64 states takes 482 us, four times the 123 of 16.

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

// Floats of LDS through which the waves add their gradients of B and C: eight units of
// four values a lane from each.
constexpr int kSwap = kGradWaves * kGradWaves * 64 * 4;

inline size_t backward_lds(int NP, int T, int set) {
    return ((size_t)2 * NP * 16 * T + kGradWaves * 3 * 16 * T + (size_t)3 * set * NP +
            (size_t)10 * set + kSwap) * 4;
}

// The sums over a row's lanes of four values: that of value s in lanes 4 s to 4 s + 3.
// Lanes change halves with their mirror image, each keeping one of two values.
template <int CTRL>
__device__ inline float dpp(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(
                                         0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ inline float row_sum4(float v0, float v1, float v2, float v3, int lane) {
    const bool hi = lane & 8, odd = lane & 4;
    const float h0 = (hi ? v2 : v0) + dpp<0x140>(hi ? v0 : v2);   // row_mirror
    const float h1 = (hi ? v3 : v1) + dpp<0x140>(hi ? v1 : v3);
    float u = (odd ? h1 : h0) + dpp<0x141>(odd ? h0 : h1);        // row_half_mirror
    u += dpp<0xb1>(u);                                            // the neighbours of a quad
    return u + dpp<0x4e>(u);
}

template <typename E, int T, int S>
__global__ __launch_bounds__(64 * kGradWaves) void scan_backward_kernel(GradArgs ga) {
    constexpr int P = 16 * T, I = T / 4, TH = 64 * kGradWaves;
    constexpr int NP = 4 * S;                      // states with those that fill the rows
    const ScanArgs &a = ga.f;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    float *tb = lds, *tc = tb + NP * P;
    float *pre = tc + NP * P;                      // delta, delta x, dy of a wave's channel
    float *swp = pre + kGradWaves * 3 * P;         // the waves' gradients of B and C
    float *carry = swp + kSwap;                    // G at the part's end, set x NP
    float *As = carry + ga.set * NP;               // A log2 e
    float *dAs = As + ga.set * NP;                 // dA
    float *ps = dAs + ga.set * NP;                 // dDskip, ddt_bias by rows: set x 4 x 2
    float *vec = ps + ga.set * 8;                  // dt_bias, Dskip: set x 2
    const int tid = threadIdx.x, lane = tid & 15, rowi = (tid >> 4) & 3;
    // uniform: a wave's rows of activations have their addresses in scalar registers
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n0 = rowi * S;
    int blk = block_of();
    const int set = blk % ga.sets;
    blk /= ga.sets;
    const int grp = blk % a.G, b = blk / a.G;
    if (b >= a.B)
        return;
    const int c0 = set * ga.set;                   // the set's first channel in the group
    const int count = min(ga.set, a.Dg - c0);
    const long long first = (long long)grp * a.Dg + c0;
    const int n_pos = __builtin_amdgcn_readfirstlane(row_length(a.lengths, b, a.L));
    const int parts = (n_pos + P - 1) / P;
    for (int i = tid; i < ga.set * NP; i += TH) {
        const int c = i / NP, n = i % NP;
        const bool ok = c < count && n < a.N;
        const long long at = (first + (ok ? c : 0)) * a.N + (ok ? n : 0);
        As[i] = ok ? decay(a.A[at]) : 0.0f;
        carry[i] = ok && ga.dstate_out ? ga.dstate_out[(long long)b * a.D * a.N + at] : 0.0f;
        dAs[i] = 0.0f;
    }
    for (int i = tid; i < ga.set * 8; i += TH)
        ps[i] = 0.0f;
    for (int i = tid; i < count; i += TH) {
        vec[2 * i] = a.dt_bias ? a.dt_bias[first + i] : 0.0f;
        vec[2 * i + 1] = a.Dskip ? a.Dskip[first + i] : 0.0f;
    }
    // the states that fill the rows read 0
    for (int i = tid; i < (NP - a.N) * P; i += TH)
        tb[a.N * P + i] = tc[a.N * P + i] = 0.0f;
    // the positions of a part that this lane prepares, and the wave's place for them
    const int pos = lane * T + rowi * I;
    float *mine = pre + wave * 3 * P;
    typedef typename Vec<E, I>::type Raw;
    Raw nx, nd, ng, nz;
    float nin[S];
    auto fetch = [&](int c, int part) {
        const int d = (int)first + c;
        const unsigned o = back<E, I>(part * P + pos, a.L);
        const E *gr = ga.dy.row<const E>(b, d), *zr = a.z.p ? a.z.row<const E>(b, d) : gr;
        nx = load_back<E, I>(a.x.row<const E>(b, d), o);
        nd = load_back<E, I>(a.dt.row<const E>(b, d), o);
        ng = load_back<E, I>(gr, o);
        nz = load_back<E, I>(zr, o);
        load_vec<float, S>(at(a.states + (((long long)b * a.D + d) * a.parts + part) * NP, n0), nin);
    };
    const int units = 2 * a.N * (P / kUnit);
    const bool whole = T == 8 || a.L >= kUnit;   // eight positions a lane: longer rasters
    typename Vec<E, kUnit>::type nt;
    if (parts > 0) {
        if (wave < count)
            fetch(wave, parts - 1);
        nt = load_tile<E, T>(a, b, grp, min(tid, units - 1), (parts - 1) * P, n_pos, whole);
    }
    for (int part = parts - 1; part >= 0; --part) {
        const int p0 = part * P;
        if (tid < units)
            store_tile<E, T>(a, tb, tc, tid, p0, n_pos, nt);
        for (int u = tid + TH; u < units; u += TH)
            store_tile<E, T>(a, tb, tc, u, p0, n_pos,
                             load_tile<E, T>(a, b, grp, u, p0, n_pos, whole));
        __syncthreads();
        nt = load_tile<E, T>(a, b, grp, min(tid, units - 1), max(p0 - P, 0), n_pos, whole);
        float dB[S][T], dC[S][T];
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int j = 0; j < T; ++j)
                dB[s][j] = dC[s][j] = 0.0f;
        for (int c = wave; c < count; c += kGradWaves) {
            const int d = (int)first + c, left = n_pos - p0 - pos;
            float x[I], dt[I], delta[I], slope[I], z[I], dout[I], dy[I], in[S], A2[S], end[S], dA[S];
            const float bias = vec[2 * c], skip = vec[2 * c + 1];
            if (p0 + P <= n_pos) {
                convert<E, I>(nx, x);
                convert<E, I>(nd, dt);
                convert<E, I>(ng, dout);
                convert<E, I>(nz, z);
            } else {
                settle<E, I>(nx, p0 + pos, a.L, n_pos, x);
                settle<E, I>(nd, p0 + pos, a.L, n_pos, dt);
                settle<E, I>(ng, p0 + pos, a.L, n_pos, dout);
                settle<E, I>(nz, p0 + pos, a.L, n_pos, z);
            }
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const float v = dt[i] + bias;
                slope[i] = a.softplus ? sigmoid(v) : 1.0f;
                delta[i] = keep_if(i < left, a.softplus ? softplus(v) : v);
                z[i] = a.z.p ? z[i] : 0.0f;
                dy[i] = a.z.p ? dout[i] * silu(z[i]) : dout[i];
                float *q = mine + slot_at<T>(pos + i);
                q[0] = delta[i];
                q[P] = delta[i] * x[i];
                q[2 * P] = dy[i];
            }
            float *own = carry + c * NP + n0;
            lds_load<S>(As + c * NP + n0, A2);
            lds_load<S>(own, end);
#pragma unroll
            for (int s = 0; s < S; ++s) {
                in[s] = n0 + s < a.N ? nin[s] : 0.0f;
                // before the next loads: behind them it would wait for them
                asm volatile("" : "+v"(in[s]));
            }
            // the next channel's, under way
            const bool more = c + kGradWaves < count;
            fetch(more ? c + kGradWaves : wave, more ? part : max(part - 1, 0));
            wave_exchange();
            float de[T], dx[T], g[T], gB[T], sA[T], yv[T], sum = 0.0f;
#pragma unroll
            for (int j = 0; j < T; j += 4) {
                const float *q = mine + (j * 4 + lane) * 4;
                lds_load<4>(q, de + j);
                lds_load<4>(q + P, dx + j);
                lds_load<4>(q + 2 * P, g + j);
            }
            wave_exchange();
#pragma unroll
            for (int j = 0; j < T; ++j) {
                sum += de[j];
                gB[j] = sA[j] = yv[j] = 0.0f;
            }
#pragma unroll
            for (int s = 0; s < S; ++s) {
                float av[T], h[T], Bv[T], Cv[T];
#pragma unroll
                for (int j = 0; j < T; j += 4) {
                    lds_load<4>(tb + tile_at<T>(n0 + s, j / 4, lane), Bv + j);
                    lds_load<4>(tc + tile_at<T>(n0 + s, j / 4, lane), Cv + j);
                }
                // the run's own map of h upwards, and of G downwards
                float e = 0.0f, f = 0.0f;
#pragma unroll
                for (int j = 0; j < T; ++j) {
                    av[j] = __builtin_amdgcn_exp2f(A2[s] * de[j]);
                    e = j ? __builtin_fmaf(av[j], e, dx[j] * Bv[j]) : dx[j] * Bv[j];
                }
#pragma unroll
                for (int j = T - 1; j >= 0; --j)
                    f = av[j] * (j < T - 1 ? __builtin_fmaf(Cv[j], g[j], f) : Cv[j] * g[j]);
                float up = __builtin_amdgcn_exp2f(A2[s] * sum), down = up;
                scan_both(up, e, down, f);
                const float start = neighbour<kFromLower>(in[s], __builtin_fmaf(up, in[s], e));
                const float low = __builtin_fmaf(down, end[s], f);
                float G = neighbour<kFromUpper>(end[s], low);
                end[s] = low;
                float prev = start;
#pragma unroll
                for (int j = 0; j < T; ++j)
                    prev = h[j] = __builtin_fmaf(av[j], prev, dx[j] * Bv[j]);
                dA[s] = 0.0f;
#pragma unroll
                for (int j = T - 1; j >= 0; --j) {
                    const float gt = __builtin_fmaf(Cv[j], g[j], G);
                    G = av[j] * gt;
                    dC[s][j] = __builtin_fmaf(g[j], h[j], dC[s][j]);
                    dB[s][j] = __builtin_fmaf(gt, dx[j], dB[s][j]);
                    gB[j] = __builtin_fmaf(gt, Bv[j], gB[j]);
                    yv[j] = __builtin_fmaf(Cv[j], h[j], yv[j]);
                    const float t = G * (j ? h[j ? j - 1 : 0] : start);
                    sA[j] = __builtin_fmaf(A2[s], t, sA[j]);
                    dA[s] = __builtin_fmaf(de[j], t, dA[s]);
                }
                // one state's values at a time: sums put off to the end would keep every
                // state's h and g in registers
#pragma unroll
                for (int j = 0; j < T; ++j)
                    asm volatile("" : "+v"(dB[s][j]), "+v"(dC[s][j]), "+v"(gB[j]), "+v"(sA[j]),
                                 "+v"(yv[j]), "+v"(dA[s]));
            }
            if (lane == 0)
                lds_store<S>(own, end);
#pragma unroll
            for (int s = 0; s < S; s += 4) {
                const float u = row_sum4(dA[s], s + 1 < S ? dA[s + 1 < S ? s + 1 : 0] : 0.0f,
                                         s + 2 < S ? dA[s + 2 < S ? s + 2 : 0] : 0.0f,
                                         s + 3 < S ? dA[s + 3 < S ? s + 3 : 0] : 0.0f, lane);
                if ((lane & 3) == 0 && s + (lane >> 2) < S)
                    dAs[c * NP + n0 + s + (lane >> 2)] += u;
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
            E *xo = ga.dx.row<E>(b, d) + p0, *to = ga.ddt.row<E>(b, d) + p0;
            E *zo = a.z.p ? ga.dz.row<E>(b, d) + p0 : nullptr;
            if (p0 + P <= a.L) {
                store_vec<E, I>(at(xo, pos), ox);
                store_vec<E, I>(at(to, pos), ot);
                if (zo)
                    store_vec<E, I>(at(zo, pos), oz);
            } else {
                store_upto<E, I>(at(xo, pos), room, ox);
                store_upto<E, I>(at(to, pos), room, ot);
                if (zo)
                    store_upto<E, I>(at(zo, pos), room, oz);
            }
            const float u = row_sum4(sD, sb, 0.0f, 0.0f, lane);
            if ((lane & 3) == 0 && lane < 8)
                ps[(c * 4 + rowi) * 2 + (lane >> 2)] += u;
        }
        // dB and dC of the part: four values a lane at a time, eight such units in LDS from
        // every wave, of which each wave adds one over the waves, in their order
        const long long rows = (long long)a.G * a.N;
#pragma unroll
        for (int u0 = 0; u0 < S * T / 4; u0 += kGradWaves) {
            constexpr int U = S * T / 4 < kGradWaves ? S * T / 4 : kGradWaves;
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                float4 *q = (float4 *)swp + (tid & 63);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int s = 4 * (u0 + u) / T, j = 4 * (u0 + u) % T;
                    const float *v = which ? &dC[s][j] : &dB[s][j];
                    q[(wave * U + u) * 64] = make_float4(v[0], v[1], v[2], v[3]);
                }
                __syncthreads();
                if (wave < U) {
                    float4 sum = q[wave * 64];
#pragma unroll
                    for (int k = 1; k < kGradWaves; ++k) {
                        const float4 v = q[(k * U + wave) * 64];
                        sum.x += v.x;
                        sum.y += v.y;
                        sum.z += v.z;
                        sum.w += v.w;
                    }
                    const int n = n0 + 4 * (u0 + wave) / T;
                    const int t0 = p0 + lane * T + 4 * (u0 + wave) % T;
                    if (n < a.N) {
                        const long long r = (((long long)which * ga.sets + set) * a.B + b) * rows +
                                            (long long)grp * a.N + n;
                        const float v[4] = {sum.x, sum.y, sum.z, sum.w};
                        store_upto<float, 4>(ga.shared + r * a.L + t0, a.L - t0, v);
                    }
                }
                __syncthreads();
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
        const int at = i / a.N * NP + i % a.N;
        out[first * a.N + i] = dAs[at];
        if (ga.dstate)
            ga.dstate[((long long)b * a.D + first) * a.N + i] = carry[at];
    }
    for (int i = tid; i < count * 2; i += TH) {
        const float *q = ps + i / 2 * 8 + i % 2;
        out[(long long)a.D * (a.N + i % 2) + first + i / 2] = (q[0] + q[2]) + (q[4] + q[6]);
    }
}

// dB and dC: the sets' sums in order, eight loads in flight a thread: bound by memory (64
// sets' sums of 4 x 16 x 4096, 134 MB: 22 us, and 39 with one load at a time).
template <typename E>
__global__ __launch_bounds__(256) void shared_sum_kernel(GradArgs ga, Rows dB, Rows dC) {
    const ScanArgs &a = ga.f;
    const int rows = a.G * a.N;
    const long long tiles = (a.L + 1023) / 1024, all = 2 * tiles * rows * a.B;
    const long long step = (long long)a.B * rows * a.L;
    for (long long unit = blockIdx.x; unit < all; unit += gridDim.x) {
        const long long tile = unit % tiles, row = unit / tiles;
        const int r = (int)(row % rows), b = (int)(row / rows % a.B);
        const int which = (int)(row / rows / a.B);
        const int t0 = (int)(tile * 1024 + threadIdx.x * 4);
        if (t0 >= a.L)
            continue;
        const int n_pos = row_length(a.lengths, b, a.L);
        float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        const float *p = ga.shared + which * ga.sets * step + ((long long)b * rows + r) * a.L + t0;
        for (int k0 = 0; k0 < ga.sets; k0 += 8) {
            float v[8][4];   // in flight together
#pragma unroll
            for (int k = 0; k < 8; ++k)
                load_upto<float, 4>(p + min(k0 + k, ga.sets - 1) * step, n_pos - t0, v[k]);
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    s[i] += k0 + k < ga.sets ? v[k][i] : 0.0f;
        }
        store_upto<E, 4>((which ? dC : dB).row<E>(b, r) + t0, a.L - t0, s);
    }
}

// dA, dDskip, ddt_bias: the batch rows' sums, eight groups in turn, then in order (5 us
// for 4 rows of 2048 channels, N = 16).
__global__ __launch_bounds__(256) void param_sum_kernel(GradArgs ga, float *dA, float *dD,
                                                        float *db) {
    __shared__ float red[8][33];
    const ScanArgs &a = ga.f;
    const long long n = (long long)a.D * (a.N + 2);
    const int l = threadIdx.x & 31, g = threadIdx.x >> 5;
    const long long i = block_of() * 32ll + l;
    float s = 0.0f;
    if (i < n)
        for (int b = g; b < a.B; b += 64) {
            float v[8];   // in flight together
#pragma unroll
            for (int k = 0; k < 8; ++k)
                v[k] = ga.params[min(b + 8 * k, a.B - 1) * n + i];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                s += b + 8 * k < a.B ? v[k] : 0.0f;
        }
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

constexpr int kStepThreads = 256;

// Q lanes a channel, four states each at a time: a state is read and written once, 16
// bytes a lane.  100 x 1024 in fp32, N = 16: 5.7 us in a graph (bytes: 3.1), the rest a
// launch and the way from the slot to its state.
template <typename E, int Q>
__global__ __launch_bounds__(kStepThreads) void scan_step_kernel(StepArgs a) {
    const int q = threadIdx.x % Q;
    const long long d0 = block_of() * (long long)(kStepThreads / Q) + threadIdx.x / Q;
    const bool live = d0 < a.D;
    const int d = live ? (int)d0 : 0, grp = d / a.Dg;
    for (int b = blockIdx.z; b < a.B; b += gridDim.z) {
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
           N <= FINC_MAX_STATE && G >= 1 && D % G == 0 && (long long)B * D < (1ll << 31) - 256 &&
           (long long)B * G * N < (1ll << 31) && (long long)G * N < (1ll << 31);
}

// Positions of a raster that the short form takes, however many rows there are: the bits
// do not depend on them.  In us, here and by the scan over lanes: 64 positions of 64 x
// 2048 channels 47 and 137, of 4 x 1024 12 and 7; 32 of those 7.2 and 8.2; but 128 of
// them 20 and 8.
constexpr int kShort = 64;
// Positions a lane: the gradients' parts and the states' layout depend on it.  A short
// raster is one part of four a lane; more than 16 states leave the gradients' registers
// room for four.
inline int lane_positions(int L, int N) { return L <= kShort || N > 16 ? 4 : 8; }
static_assert(kShort <= 16 * 4, "one part");
// States a lane of a row in the gradients, a quarter of them all.
inline int row_states(int N) { return N <= 4 ? 1 : N <= 8 ? 2 : N <= 16 ? 4 : N <= 32 ? 8 : 16; }
inline long long part_count(int L, int N) {
    return cdivll(L > 0 ? L : 1, 16 * lane_positions(L, N));
}

template <typename E, int T>
int launch_forward(ScanArgs &c, hipStream_t s) {
    constexpr int CB = kThreads / 64;
    c.blocks = (int)cdivll(c.Dg, CB);
    const long long grid = (long long)c.blocks * c.G * c.B;
    const size_t lds =
        ((size_t)4 * c.N * 16 * T + 2 * CB * c.N + CB * 2 * 16 * T) * sizeof(float);
    if (grid >= (1ll << 31) || lds > (size_t)kLds)
        return FINC_EUNSUPPORTED;
    if (lds > 64 * 1024)
        (void)hipFuncSetAttribute((const void *)scan_forward_kernel<E, T>,
                                  hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    (void)hipGetLastError();   // the launch check decides
    hipLaunchKernelGGL((scan_forward_kernel<E, T>), grid_of(grid), dim3(kThreads),
                       (unsigned)lds, s, c);
    return launched();
}

template <typename E, int S, bool ALL>
int launch_short(ScanArgs &c, hipStream_t s) {
    // a wave a workgroup where whole ones would leave compute units without work
    const int threads =
        (long long)c.B * c.D >= 1024ll * kShortThreads / 4 ? kShortThreads : 64;
    c.blocks = (int)cdivll(c.Dg, threads / 4);
    const long long grid = (long long)c.blocks * c.G * c.B;
    static_assert(2 * 4 * 16 * kShort * sizeof(float) <= 64 * 1024, "B and C in LDS");
    const size_t lds = (size_t)2 * 4 * S * cdivll(c.L, 16) * 16 * sizeof(float);
    if (grid >= (1ll << 31))
        return FINC_EUNSUPPORTED;
    (void)hipGetLastError();   // the launch check decides
    hipLaunchKernelGGL((scan_short_kernel<E, S, ALL>), grid_of(grid), dim3(threads),
                       (unsigned)lds, s, c);
    return launched();
}
template <typename E, int S>
int launch_short(ScanArgs &c, hipStream_t s) {
    return c.N == 4 * S ? launch_short<E, S, true>(c, s) : launch_short<E, S, false>(c, s);
}
template <typename E>
int dispatch_short(ScanArgs &c, hipStream_t s) {
    const int S = row_states(c.N);
    return S == 1   ? launch_short<E, 1>(c, s)
           : S == 2 ? launch_short<E, 2>(c, s)
           : S == 4 ? launch_short<E, 4>(c, s)
           : S == 8 ? launch_short<E, 8>(c, s)
                    : launch_short<E, 16>(c, s);
}

// The parts of the arguments that both directions use.
void scan_common(const finc_scan_args *a, ScanArgs &c) {
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
    c.NP = 4 * row_states(a->N);
}

// Channels of a set: a workgroup a compute unit where there are that many channels,
// and at most 64, which the state in LDS holds.
inline int set_channels(int B, int D, int G) {
    long long c = cdivll(cdivll((long long)B * D, 256), kGradWaves) * kGradWaves;
    const long long most = cdivll(D / G, kGradWaves) * kGradWaves;
    c = c < most ? c : most;
    return (int)(c < kGradWaves ? kGradWaves : c > 64 ? 64 : c);
}

template <typename E, int T, int S>
int launch_backward(GradArgs &c, hipStream_t s) {
    const long long grid = (long long)c.sets * c.f.G * c.f.B;
    const size_t lds = backward_lds(4 * S, T, c.set);
    if (grid >= (1ll << 31) || lds > (size_t)kLds)
        return FINC_EUNSUPPORTED;
    (void)hipFuncSetAttribute((const void *)scan_backward_kernel<E, T, S>,
                              hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    (void)hipGetLastError();   // the launch check decides
    hipLaunchKernelGGL((scan_backward_kernel<E, T, S>), grid_of(grid), dim3(64 * kGradWaves),
                       (unsigned)lds, s, c);
    return launched();
}

template <typename E>
int dispatch_backward(GradArgs &c, hipStream_t s) {
    const int S = row_states(c.f.N);
    if (lane_positions(c.f.L, c.f.N) == 4)
        return S == 1   ? launch_backward<E, 4, 1>(c, s)
               : S == 2 ? launch_backward<E, 4, 2>(c, s)
               : S == 4 ? launch_backward<E, 4, 4>(c, s)
               : S == 8 ? launch_backward<E, 4, 8>(c, s)
                        : launch_backward<E, 4, 16>(c, s);
    return S == 1   ? launch_backward<E, 8, 1>(c, s)
           : S == 2 ? launch_backward<E, 8, 2>(c, s)
                    : launch_backward<E, 8, 4>(c, s);
}

// A buffer of a * b * c * d floats, whole 256-byte lines; 0 for one of more bytes than
// an address space has.
inline size_t floats(long long a, long long b, long long c, long long d) {
    const unsigned __int128 n = (unsigned __int128)a * b * c * d;
    return n >> 48 ? 0 : ((size_t)n * 4 + 255) / 256 * 256;
}
inline size_t shared_bytes(int B, int D, int L, int N, int G) {
    return floats(2 * cdivll(D / G, set_channels(B, D, G)), B, (long long)G * N, L);
}
// Whether both of the gradients' buffers have a size.
inline bool grad_sizes(int B, int D, int L, int N, int G) {
    return B == 0 || L == 0 || (shared_bytes(B, D, L, N, G) && floats(B, D, N + 2, 1));
}

}  // namespace

extern "C" {

size_t finc_selective_scan_states_bytes(int B, int D, int L, int N) {
    if (!scan_shape(FINC_F32, B, D, L, N, 1))
        return 0;
    return floats(B, D, part_count(L, N), 4 * row_states(N));
}

int finc_selective_scan_forward(const finc_scan_args *a, hipStream_t stream) {
    if (!a || !scan_shape(a->type, a->B, a->D, a->L, a->N, a->G) || ((uintptr_t)a->states & 255u))
        return FINC_EINVAL;
    const int sz = type_size(a->type), B = a->B, D = a->D, L = a->L;
    if (a->states && B > 0 && !finc_selective_scan_states_bytes(B, D, L, a->N))
        return FINC_EUNSUPPORTED;
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
    with_type(a->type, [&](auto e) {
        typedef decltype(e) E;
        rc = L <= kShort                    ? dispatch_short<E>(c, stream)
             : lane_positions(L, a->N) == 4 ? launch_forward<E, 4>(c, stream)
                                            : launch_forward<E, 8>(c, stream);
    });
    return rc;
}

size_t finc_selective_scan_workspace_bytes(int B, int D, int L, int N, int G) {
    if (!scan_shape(FINC_F32, B, D, L, N, G) || !grad_sizes(B, D, L, N, G))
        return 0;
    return shared_bytes(B, D, L, N, G) + floats(B, D, N + 2, 1);
}

int finc_selective_scan_backward(const finc_scan_args *a, const finc_scan_grads *g,
                                 hipStream_t stream) {
    if (!a || !g || !scan_shape(a->type, a->B, a->D, a->L, a->N, a->G) || !g->dA ||
        ((uintptr_t)a->states & 255u) || ((uintptr_t)g->workspace & 255u))
        return FINC_EINVAL;
    const int sz = type_size(a->type), B = a->B, D = a->D, L = a->L, N = a->N, G = a->G;
    if (!grad_sizes(B, D, L, N, G) || (B > 0 && !finc_selective_scan_states_bytes(B, D, L, N)))
        return FINC_EUNSUPPORTED;
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
    const long long params = cdivll((long long)D * (N + 2), 32);
    if (params > (1ll << 31))
        return FINC_EUNSUPPORTED;
    if (B > 0) {
        with_type(a->type, [&](auto e) { rc = dispatch_backward<decltype(e)>(c, stream); });
        if (rc != FINC_OK)
            return rc;
    }
    if (sums > 0) {
        with_type(a->type, [&](auto e) {
            const unsigned blocks = sums < (1 << kRowBits) ? (unsigned)sums : 1u << kRowBits;
            hipLaunchKernelGGL(shared_sum_kernel<decltype(e)>, dim3(blocks), dim3(256), 0, stream,
                               c, rows_of(g->dBm), rows_of(g->dCm));
        });
        rc = launched();
        if (rc != FINC_OK)
            return rc;
    }
    hipLaunchKernelGGL(param_sum_kernel, grid_of(params), dim3(256), 0, stream, c, g->dA,
                       g->dDskip, g->ddt_bias);
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
                          flat(a->state, elements(a->S, D, a->N), 4)};
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
        dim3 grid = grid_of(cdivll(D, a->N <= 4 ? kStepThreads : kStepThreads / 4));
        grid.z = (unsigned)(B < 32768 ? B : 32768);
        if (a->N <= 4)
            hipLaunchKernelGGL((scan_step_kernel<E, 1>), grid, dim3(kStepThreads), 0, stream, c);
        else
            hipLaunchKernelGGL((scan_step_kernel<E, 4>), grid, dim3(kStepThreads), 0, stream, c);
    });
    return launched();
}

}  // extern "C"
