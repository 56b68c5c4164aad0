// Operands of the gated delta rule's kernels: 16x16 products of a wave, and their operands.
//
// A product D [16 x 16] += A [16 x SL] B [SL x 16] has, lane l = 16 g + n: D rows 4 g + j in register j, column n; A row n and B column n, contraction indices
// FE g + e in element e (fp16: SL = 32, eight elements; fp32: SL = 16, four elements, one instruction each).  Results become the B operand of the next product in
// place: rows along the registers are its contraction index.  For fp16 that takes two tiles for a slab of 32, and their rows are chosen such that a lane's eight
// registers are eight successive indices: row m of tile t is index
//     delta_row(t, m) = 32 (t / 2) + 8 (m / 4) + 4 (t % 2) + m % 4          (fp32: 16 t + m).
//
// With bf16 tensors the operands are fp16: q, k and what is computed from them as they are, and what hangs on v (states, U; backwards d_o, their gradients) over a power of two that
// puts the largest finite value of the first state and the first chunk, per sequence, head and 16 columns, between 32 and 64 (delta_scan.hip has what follows if later ones are larger), so
// that values of any size have fp16's eleven bits (down to 2^-19 of the largest; less below).  What is computed is multiplied as the sum of NP = 2 fp16 numbers, the second
// the rounding of what the first leaves (relative steps of 2^-23; o and gradients 2e-7 of their norm from 64 bits before they are rounded).  Single ones (2^-12) are rounded relative to the state and to P's
// rows, not to a step of a token: 4e-4 of the norm over random keys and betas below 1, but 5e-3, three times bf16's own rounding, over keys whose products are 0.95 with betas near 2, and more the longer a
// chunk's steps cancel.  (They took 304 us where two take 388: forward of 4 x 16 heads, 8192 tokens.  Sums of bf16 numbers need three for as much: states 331 us of 737 in all.)
#pragma once
#include "delta_decl.h"

namespace path {

template <typename T> struct DeltaOps;
template <> struct DeltaOps<half_t> {
    static constexpr int SL = 32, FE = 8, TPS = 2;      // contraction indices of a slab, elements of a fragment, result tiles that make a slab
    static constexpr int NP = 2;                        // numbers that an operand is the sum of
    static constexpr int NLOW = 6;                      // fragments of a 64 x 64 lower (or upper) triangular operand
    typedef halfx8 Frag;
    static __device__ __forceinline__ f32x4 mma(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ int row(int t, int m) { return 32 * (t >> 1) + 8 * (m >> 2) + 4 * (t & 1) + (m & 3); }
    static constexpr __device__ __forceinline__ bool low(int t, int s) { return s <= t >> 1; }
    static constexpr __device__ __forceinline__ int low_at(int t, int s) { return t < 2 ? t : 2 * (t - 1) + s; }              // t >= 2: slabs 0, 1
    static constexpr __device__ __forceinline__ bool up(int t, int s) { return s >= t >> 1; }
    static constexpr __device__ __forceinline__ int up_at(int t, int s) { return t < 2 ? 2 * t + s : 2 + t; }                 // t < 2: slabs 0, 1
};
template <> struct DeltaOps<float> {
    static constexpr int SL = 16, FE = 4, TPS = 1, NP = 1, NLOW = 10;
    typedef f32x4 Frag;
    static __device__ __forceinline__ f32x4 mma(Frag a, Frag b, f32x4 c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ int row(int t, int m) { return 16 * t + m; }
    static constexpr __device__ __forceinline__ bool low(int t, int s) { return s <= t; }
    static constexpr __device__ __forceinline__ int low_at(int t, int s) { return t * (t + 1) / 2 + s; }
    static constexpr __device__ __forceinline__ bool up(int t, int s) { return s >= t; }
    static constexpr __device__ __forceinline__ int up_at(int t, int s) { return 4 * t - t * (t - 1) / 2 + s - t; }
};

template <typename T, int NP> struct DeltaParts { typename DeltaOps<T>::Frag p[NP]; };

// x as a sum of NP numbers of type T (fp32: itself)
template <typename T, int NP> __device__ __forceinline__ void delta_split(const float* x, DeltaParts<T, NP>& o) {
    constexpr int FE = DeltaOps<T>::FE;
    float r[FE];
#pragma unroll
    for (int e = 0; e < FE; ++e) r[e] = x[e];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
#pragma unroll
        for (int e = 0; e < FE; ++e) o.p[p][e] = (T)r[e];
        if (p + 1 < NP) {
#pragma unroll
            for (int e = 0; e < FE; ++e) r[e] -= (float)o.p[p][e];
        }
    }
}
// four numbers as sums of NP fp16 numbers each, two to a register
template <int NP> struct DeltaSplit4 {
    uint2 p[NP];
    __device__ __forceinline__ explicit DeltaSplit4(const f32x4& v) {
        f32x4 r = v;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const halfx4 h = __builtin_convertvector(r, halfx4);
            p[i] = __builtin_bit_cast(uint2, h);
            if (i + 1 < NP) r = r - __builtin_convertvector(h, f32x4);
        }
    }
};
// eight values of the caller's type as an operand
__device__ __forceinline__ halfx8 delta_operand(const bf16x8& f) {
    typedef float f32x8 __attribute__((ext_vector_type(8)));
    return __builtin_convertvector(__builtin_convertvector(f, f32x8), halfx8);
}
__device__ __forceinline__ f32x4 delta_operand(const f32x4& f) { return f; }
// c += a b, products of parts that together are below the last one left out
template <typename T, int NA, int NB> __device__ __forceinline__ f32x4 delta_mma(const DeltaParts<T, NA>& a, const DeltaParts<T, NB>& b, f32x4 c) {
    constexpr int NP = NA > NB ? NA : NB;
#pragma unroll
    for (int i = NA - 1; i >= 0; --i)      // (small ones first)
#pragma unroll
        for (int j = NB - 1; j >= 0; --j)
            if (i + j < NP) c = DeltaOps<T>::mma(a.p[i], b.p[j], c);
    return c;
}

// K in LDS: 64 rows of D elements without padding, the 16-byte pieces of a row permuted by an exclusive or with a number made of the row, so that neither a fragment along the
// rows (sixteen rows' pieces of one column) nor a transposing read (four rows, four pieces) meets itself on a bank.
template <typename C, int D> struct DeltaTile {
    static constexpr int ROWB = D * (int)sizeof(C), PPR = ROWB / 16, BYTES = 64 * ROWB;
    static __device__ __forceinline__ int turn(int row) {
        return sizeof(C) == 4 ? row & 15 : D == 128 ? ((row & 3) << 2) | ((row >> 3) & 3) : (((row >> 1) & 1) << 2) | ((row >> 3) & 3);
    }
    static __device__ __forceinline__ int piece(int row, int p) { return row * ROWB + ((p ^ turn(row)) << 4); }
};
// four rows of a column, as a transposing read gives them to the lane that asks for the row and the four columns of its number
__device__ __forceinline__ halfx4 delta_ld_tr(const unsigned char* p) {
    typedef short v4s __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(halfx4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)p));
}

// the exponent that puts numbers up to m between 32 and 64 (2^100 and 2^-100 are the ends)
__device__ __forceinline__ int delta_exponent(float m) {
    const int e = (int)(__float_as_uint(m) >> 23) - 127 - 5;
    return e < -100 ? -100 : e > 100 ? 100 : e;
}
__device__ __forceinline__ float delta_power(int e) { return __uint_as_float((unsigned)(127 + e) << 23); }
__device__ __forceinline__ float delta_finite(float x) { const float y = fabsf(x); return __float_as_uint(y) < 0x7f800000u ? y : 0.f; }

}  // namespace path
