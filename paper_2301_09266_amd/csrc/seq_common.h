// seq_common.h -- what the sequence operators (causal_conv.hip,
// selective_scan.hip, add_norm.hip) share: activation types, loads and stores
// of any alignment, reductions over lanes, and the host's argument checks.
#ifndef FINC_SEQ_COMMON_H
#define FINC_SEQ_COMMON_H

#include <hip/hip_runtime.h>

#include <stddef.h>
#include <stdint.h>

#include "device_common.h"
#include "finc.h"

namespace finc_seq {

using finc_detail::FastDiv;
using finc_detail::fdiv;
using finc_detail::make_fastdiv;

typedef __bf16 bf16;
typedef _Float16 f16;

// ---- loads and stores ---------------------------------------------------------
// Rows may start at any multiple of the element's size (odd lengths, views): the
// vectors are declared with the element's alignment, which global loads and
// stores of up to 16 bytes take as they are.

template <typename E, int N>
struct Vec {
    typedef E type __attribute__((ext_vector_type(N), aligned(sizeof(E))));
};

// Elements a 16-byte access holds.
template <typename E>
constexpr int kPer16 = 16 / (int)sizeof(E);

template <typename E, int N>
__device__ inline void load_vec(const E *p, float *v) {
    constexpr int C = N < kPer16<E> ? N : kPer16<E>;
    static_assert(N % C == 0, "whole accesses");
#pragma unroll
    for (int i = 0; i < N; i += C) {
        const typename Vec<E, C>::type t = *(const typename Vec<E, C>::type *)(p + i);
#pragma unroll
        for (int j = 0; j < C; ++j)
            v[i + j] = (float)t[j];
    }
}

// The value, of which the compiler knows nothing: what follows from it is formed here
// and not ahead of a loop, where the addresses and masks of a vector's elements would
// take its registers for a path that few lanes take.
__device__ inline int afresh(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// The first `count` (any int) of N elements; the others are 0.  A part of a vector
// takes its elements one by one, the last one again in place of those past it: no
// branch an element.
template <typename E, int N>
__device__ inline void load_upto(const E *p, int count, float *v) {
    if (count >= N) {
        load_vec<E, N>(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        v[i] = 0.0f;
    if (count > 0) {
        const int n = afresh(count);
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = (float)p[min(i, n - 1)];
#pragma unroll
        for (int i = 1; i < N; ++i)
            v[i] = i < n ? v[i] : 0.0f;
    }
}

template <typename E, int N>
__device__ inline void store_vec(E *p, const float *v) {
    constexpr int C = N < kPer16<E> ? N : kPer16<E>;
#pragma unroll
    for (int i = 0; i < N; i += C) {
        typename Vec<E, C>::type t;
#pragma unroll
        for (int j = 0; j < C; ++j)
            t[j] = (E)v[i + j];
        *(typename Vec<E, C>::type *)(p + i) = t;
    }
}

// The first n < N of N elements, N a power of two.
template <typename E, int N>
__device__ inline void store_bits(E *p, int n, const float *v) {
    if constexpr (N > 1) {
        constexpr int H = N / 2;
        float u[H];
#pragma unroll
        for (int i = 0; i < H; ++i)
            u[i] = v[i];
        if (n & H) {
            store_vec<E, H>(p, v);
            p += H;
#pragma unroll
            for (int i = 0; i < H; ++i)
                u[i] = v[i + H];
        }
        store_bits<E, H>(p, n, u);
    }
}
template <typename E, int N>
__device__ inline void store_upto(E *p, int count, const float *v) {
    if (count >= N) {
        store_vec<E, N>(p, v);
        return;
    }
    // a half, a quarter and so on, each where the count has it
    const int n = afresh(count);
    if (n > 0)
        store_bits<E, N>(p, n, v);
}

// ---- activations ----------------------------------------------------------------
// exp2 and the reciprocal are the hardware's (1 ulp each).

__device__ inline float exp_fast(float v) {
    return __builtin_amdgcn_exp2f(v * 1.44269504088896341f);
}
__device__ inline float sigmoid(float v) {
    // 1 / (1 + inf) = 0 on the left, 1 / (1 + 0) = 1 on the right
    return __builtin_amdgcn_rcpf(1.0f + exp_fast(-v));
}
// An infinite v times a sigmoid of 0 has no value: v stays within 1e30 of 0.  (The
// maximum and the median drop NaN, which the sigmoid brings back.)
__device__ inline float silu(float v) { return __builtin_fmaxf(v, -1e30f) * sigmoid(v); }
// d silu / dv, with sg = sigmoid(v).
__device__ inline float silu_grad(float v, float sg) {
    return sg * __builtin_fmaf(__builtin_amdgcn_fmed3f(v, -1e30f, 1e30f), 1.0f - sg, 1.0f);
}
// v, or 0: a mask of bits, so that what v takes to compute gets no branch.
__device__ inline float keep_if(bool ok, float v) {
    return __builtin_bit_cast(float, __builtin_bit_cast(int, v) & -(int)ok);
}
// log(1 + e^v) = max(v, 0) + log1p(e^-|v|).  The logarithm is 2 atanh(s), s = e / (2 +
// e) <= 1/3, by a Chebyshev fit of atanh(s) / s in s^2 on [0, 1/9] (relative error
// 4e-9), and small e keeps its relative precision, which the logarithm of 1 + e loses.
__device__ inline float softplus(float v) {
    const float e = exp_fast(-__builtin_fabsf(v));
    const float s = e * __builtin_amdgcn_rcpf(2.0f + e), q = s * s;
    float p = 0.14087328633621787f;
    p = __builtin_fmaf(p, q, 0.139807094169866f);
    p = __builtin_fmaf(p, q, 0.20012426861758947f);
    p = __builtin_fmaf(p, q, 0.3333315796754006f);
    p = __builtin_fmaf(p, q, 1.0000000039388746f);
    // NaN comes through e: the maximum alone would drop it
    return __builtin_fmaf(2.0f * s, p, __builtin_fmaxf(v, 0.0f));
}

// Between what a wave's lanes write to LDS and what others of them read of it, and before
// they write there again.  The LDS takes a wave's accesses in order: what is needed is that
// the compiler keeps that order, which the barrier alone does not ask of it.
__device__ inline void wave_exchange() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// ---- reductions over lanes -------------------------------------------------------

template <int CTRL>
__device__ inline float dpp_zero(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(
                                         0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// The sum over a row of 16 lanes, in its last lane.
__device__ inline float row_sum(float v) {
    v += dpp_zero<0x118>(v);   // row_shr:8
    v += dpp_zero<0x114>(v);
    v += dpp_zero<0x112>(v);
    v += dpp_zero<0x111>(v);
    return v;
}
// The sum over the wave, in every lane (a scalar register).
__device__ inline float wave_sum(float v) {
    v = row_sum(v);
    v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x142,
                                                               0xa, 0xf, false));   // row_bcast:15
    v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x143,
                                                               0xc, 0xf, false));   // row_bcast:31
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// ---- grids -------------------------------------------------------------------------
// A launch holds fewer than 2^32 threads in x: more workgroups than 2^21 lie in rows of
// y, the last of which may hold some without work.

constexpr int kRowBits = 21;
inline dim3 grid_of(long long blocks) {   // up to 2^31
    const long long row = 1ll << kRowBits;
    return blocks <= row ? dim3((unsigned)blocks)
                         : dim3((unsigned)row, (unsigned)((blocks + row - 1) / row));
}
__device__ inline int block_of() { return (int)(blockIdx.y << kRowBits | blockIdx.x); }

// ---- the host's checks -------------------------------------------------------------

inline int launched() { return hipGetLastError() == hipSuccess ? FINC_OK : FINC_EHIP; }
inline long long cdivll(long long a, long long b) { return (a + b - 1) / b; }

inline int type_size(int type) {
    return type == FINC_F32 ? 4 : type == FINC_BF16 || type == FINC_F16 ? 2 : 0;
}

// A buffer's region: `outer` blocks `so` elements apart of `inner` rows `si`
// apart of `n` elements of `size` bytes.
struct Region {
    const void *p;
    long long outer, so, inner, si, n;
    int size;
};
// a b c, or a length that no region has.
inline long long elements(long long a, long long b, long long c) {
    long long n;
    return __builtin_mul_overflow(a, b, &n) || __builtin_mul_overflow(n, c, &n) ? INT64_MAX : n;
}
inline Region flat(const void *p, long long n, int size) { return {p, 1, 0, 1, 0, n, size}; }
inline Region raster(const finc_raster &r, int B, int D, int L, int size) {
    return {r.p, B, r.sb, D, r.sd, L, size};
}

// The region's extent in elements; -1 where it is negative or too far for 62 bits
// of bytes.
inline long long extent(const Region &r) {
    if (r.outer == 0 || r.inner == 0 || r.n == 0)
        return 0;
    long long a, b, e;
    if (r.so < 0 || r.si < 0 || __builtin_mul_overflow(r.outer - 1, r.so, &a) ||
        __builtin_mul_overflow(r.inner - 1, r.si, &b) || __builtin_add_overflow(a, b, &e) ||
        __builtin_add_overflow(e, r.n, &e) || e > (1ll << 59))
        return -1;
    return e;
}

// An input: any strides of 0 and more; present and aligned to its elements
// unless empty.
inline bool readable(const Region &r) {
    const long long e = extent(r);
    return e == 0 || (e > 0 && r.p && (uintptr_t)r.p % r.size == 0);
}
// An output: no two of its elements share an address, as one of its steps passes the
// rows that the other one spans.
inline bool writable(const Region &r) {
    if (!readable(r))
        return false;
    if (extent(r) == 0)
        return true;
    const long long inner = (r.inner - 1) * r.si + r.n, outer = (r.outer - 1) * r.so + r.n;
    return ((r.inner == 1 || r.si >= r.n) && (r.outer == 1 || r.so >= inner)) ||
           (r.so >= r.n && r.si >= outer);
}

// Whether two regions share memory.  Regions of the same steps whose blocks lie
// side by side in a common one (the halves of a projection) do not.
inline bool overlap(const Region &a, const Region &b) {
    const long long ea = extent(a), eb = extent(b);
    if (ea <= 0 || eb <= 0 || !a.p || !b.p)
        return false;
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    if (x >= y + (uintptr_t)eb * b.size || y >= x + (uintptr_t)ea * a.size)
        return false;
    const long long step = a.so;
    const long long ia = (a.inner - 1) * a.si + a.n, ib = (b.inner - 1) * b.si + b.n;
    if (a.size == b.size && a.so == b.so && a.outer > 1 && b.outer > 1 && ia <= step &&
        ib <= step) {
        const long long bytes = step * a.size;
        const long long off = (((long long)(y - x)) % bytes + bytes) % bytes;
        if (off >= ia * a.size && off + ib * b.size <= bytes)
            return false;
    }
    return true;
}

// Outputs against inputs and each other.
template <int NI, int NO>
inline bool disjoint(const Region (&in)[NI], const Region (&out)[NO]) {
    for (int o = 0; o < NO; ++o) {
        for (int i = 0; i < NI; ++i)
            if (overlap(out[o], in[i]))
                return false;
        for (int p = o + 1; p < NO; ++p)
            if (overlap(out[o], out[p]))
                return false;
    }
    return true;
}

// Calls f with a value of the activation type.
template <typename F>
inline void with_type(int type, F f) {
    if (type == FINC_F32)
        f(float());
    else if (type == FINC_BF16)
        f(bf16());
    else
        f(f16());
}

}  // namespace finc_seq

#endif  // FINC_SEQ_COMMON_H
