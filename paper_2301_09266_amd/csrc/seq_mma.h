// seq_mma.h -- matrix fragments of the sequence operators' products: 16 x 16 tiles
// of sums over 32 elements, from tiles in LDS.
//
// A fragment holds, in lane 16 g + m, elements k = 8 g .. 8 g + 7 of row (or column) m;
// a tile of results holds, in lane 16 g + m, rows 4 g .. 4 g + 3 of column m.
#ifndef FINC_SEQ_MMA_H
#define FINC_SEQ_MMA_H

#include "seq_common.h"

namespace finc_seq {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x4 __attribute__((ext_vector_type(4)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <typename E>
using Frag = E __attribute__((ext_vector_type(8)));

__device__ inline f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4 mma(f16x8 a, f16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
// fp32 in full: eight products of four elements, element i of every lane's eight in the
// i-th (the order of the sum is the same for both operands, which is all that it takes).
__device__ inline f32x4 mma(f32x8 a, f32x8 b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
}

// ---- fragments from LDS ----------------------------------------------------------

// Eight neighbouring elements, at a multiple of 16 bytes.
template <typename E>
__device__ inline Frag<E> frag_row(const E *p) {
    typedef E V __attribute__((ext_vector_type(8), aligned(16)));
    return *(const V *)p;
}

// Four rows `ld` apart of a lane's column, transposed by the read: each 16 lanes read 4
// rows of 16 elements, lane 4 r + c the four elements at its own address, and lane
// 4 c + i receives the i-th of column block c, one element of each row.
template <typename E>
__device__ inline s16x4 read_transposed(const E *p) {
    typedef __attribute__((address_space(3))) s16x4 *Lds;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p));
}

// The fragment of a tile whose k runs over rows `ld` apart from row 0 of p on: lane
// 16 g + 4 c + i holds rows 8 g .. 8 g + 7 of column `step` c + i.
template <int step, typename E>
__device__ inline Frag<E> frag_column(const E *p, int ld, int lane) {
    const int g = lane >> 4, m = lane & 15;
    if constexpr (sizeof(E) == 2) {
        const E *q = p + (8 * g + (m >> 2)) * ld + step * (m & 3);
        const s16x4 a = read_transposed(q), b = read_transposed(q + 4 * ld);
        const auto v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(Frag<E>, v);
    } else {
        const E *q = p + 8 * g * ld + step * (m >> 2) + (m & 3);
        Frag<E> v;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = q[i * ld];
        return v;
    }
}

// ---- sums of inputs and of fp32 values ------------------------------------------------
// The products of an input of 16 bits with an fp32 value take the value as two parts, the
// second the rest of the first.  Two bf16 parts are 16 bits of it at least (an error of
// 2^-17 of the value), with the range of fp32; a third part, the rest of both, holds all of
// it.  An fp16 input beside them is two bf16 parts itself, exactly; the smallest of its
// products is left out (2^-17).  Where values can be brought near each other by a power of
// two they are two fp16 parts beside the input as it is: 22 bits of the largest, and of
// all that are within 2^-16 of it.  In fp32 all is fp32.

typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef f16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Two values' bf16 parts: the nearest, whose halves of a register are the fp32 values that
// they stand for, and what they leave of `v`.  (Element by element the compiler rounds each
// of them a second time alone to take it back.)
__device__ inline bf16x2 part_of_two(float (&v)[2]) {
    const bf16x2 h = __builtin_convertvector((f32x2{v[0], v[1]}), bf16x2);
    const unsigned u = __builtin_bit_cast(unsigned, h);
    v[0] -= __builtin_bit_cast(float, u << 16);
    v[1] -= __builtin_bit_cast(float, u & 0xffff0000u);
    return h;
}

struct Parts {
    bf16x8 hi, lo;
};
__device__ inline Parts split(const f32x8 &v) {
    Parts p;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        float r[2] = {v[i], v[i + 1]};
        const bf16x2 a = part_of_two(r);
        const bf16x2 b = __builtin_convertvector((f32x2{r[0], r[1]}), bf16x2);
        p.hi[i] = a[0], p.hi[i + 1] = a[1];
        p.lo[i] = b[0], p.lo[i + 1] = b[1];
    }
    return p;
}
// The same with the rest of both.
__device__ inline Parts split(const f32x8 &v, bf16x8 &rest) {
    Parts p;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        float r[2] = {v[i], v[i + 1]};
        const bf16x2 a = part_of_two(r), b = part_of_two(r);
        const bf16x2 c = __builtin_convertvector((f32x2{r[0], r[1]}), bf16x2);
        p.hi[i] = a[0], p.hi[i + 1] = a[1];
        p.lo[i] = b[0], p.lo[i + 1] = b[1];
        rest[i] = c[0], rest[i + 1] = c[1];
    }
    return p;
}

struct Halves {
    f16x8 hi, lo;
};
// of values below 2^15
__device__ inline Halves halve(const f32x8 &v) {
    Halves p;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const f16x2 h = __builtin_convertvector((f32x2{v[i], v[i + 1]}), f16x2);
        unsigned u = __builtin_bit_cast(unsigned, h);
        asm("" : "+v"(u));   // both halves from the register that holds them, as above
        const f16x2 a = __builtin_bit_cast(f16x2, u);
        const f32x2 r = {v[i] - (float)a[0], v[i + 1] - (float)a[1]};
        const f16x2 b = __builtin_convertvector(r, f16x2);
        p.hi[i] = a[0], p.hi[i + 1] = a[1];
        p.lo[i] = b[0], p.lo[i + 1] = b[1];
    }
    return p;
}

// What an fp32 value is held as beside inputs of type E, and the inputs beside it: of any
// size (Value, Input), and of the state, whose columns have a scale in fp16 (Scaled,
// Beside).
template <typename E>
struct Mixed {
    typedef Parts Value;
    typedef bf16x8 Input;
    __device__ static Input input(const Frag<E> &v) { return v; }
    // a's rows by b's columns
    __device__ static f32x4 mma(const Value &a, const Input &b, f32x4 c) {
        return finc_seq::mma(a.hi, b, finc_seq::mma(a.lo, b, c));
    }
    __device__ static f32x4 mma(const Input &a, const Value &b, f32x4 c) {
        return finc_seq::mma(a, b.hi, finc_seq::mma(a, b.lo, c));
    }
    typedef Value Scaled;
    typedef Input Beside;
    __device__ static Scaled scaled(const f32x8 &v) { return split(v); }
    __device__ static Beside beside(const Frag<E> &v) { return v; }
};
template <>
struct Mixed<f16> {
    typedef Parts Value;
    typedef Parts Input;
    __device__ static Input input(const f16x8 &v) {
        return split(__builtin_convertvector(v, f32x8));
    }
    __device__ static f32x4 mma(const Parts &a, const Parts &b, f32x4 c) {
        c = finc_seq::mma(a.lo, b.hi, c);
        c = finc_seq::mma(a.hi, b.lo, c);
        return finc_seq::mma(a.hi, b.hi, c);
    }
    typedef Halves Scaled;
    typedef f16x8 Beside;
    __device__ static Scaled scaled(const f32x8 &v) { return halve(v); }
    __device__ static Beside beside(const f16x8 &v) { return v; }
    __device__ static f32x4 mma(const Halves &a, const f16x8 &b, f32x4 c) {
        return finc_seq::mma(a.hi, b, finc_seq::mma(a.lo, b, c));
    }
    __device__ static f32x4 mma(const f16x8 &a, const Halves &b, f32x4 c) {
        return finc_seq::mma(a, b.hi, finc_seq::mma(a, b.lo, c));
    }
};
template <>
struct Mixed<float> {
    typedef f32x8 Value;
    typedef f32x8 Input;
    __device__ static Input input(const f32x8 &v) { return v; }
    __device__ static f32x4 mma(const f32x8 &a, const f32x8 &b, f32x4 c) {
        return finc_seq::mma(a, b, c);
    }
    typedef f32x8 Scaled;
    typedef f32x8 Beside;
    __device__ static Scaled scaled(const f32x8 &v) { return v; }
    __device__ static Beside beside(const f32x8 &v) { return v; }
};

}  // namespace finc_seq

#endif  // FINC_SEQ_MMA_H
