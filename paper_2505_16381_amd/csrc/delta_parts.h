// Operands of the gated delta rule's kernels: 16x16 products of a wave, and their operands as sums of bf16 numbers.
//
// A product D [16 x 16] += A [16 x SL] B [SL x 16] has, lane l = 16 g + n: D rows 4 g + j in register j, column n; A row n and B column n, contraction indices
// FE g + e in element e (bf16: SL = 32, eight elements; fp32: SL = 16, four elements, one instruction each).  Results become the B operand of the next product in
// place: rows along the registers are its contraction index.  For bf16 that takes two tiles for a slab of 32, and their rows are chosen such that a lane's eight
// registers are eight successive indices: row m of tile t is index
//     delta_row(t, m) = 32 (t / 2) + 8 (m / 4) + 4 (t % 2) + m % 4          (fp32: 16 t + m).
// What is computed -- states, predictions, the chunk's matrices -- is multiplied as a sum of NP bf16 numbers, each the rounding of what the ones before it leave;
// inputs are one.  Of the products of the parts those below the last part's size are left out.  NP = 2 (relative steps of 2^-17) is enough for results that are rounded to
// bf16; NP = 3 (2^-25) where states are handed out in 32 bits: with two, states came out 4e-6 (of their norm) from 64 bits, ten times what sums in 32 bits cost.
#pragma once
#include "delta_decl.h"

namespace path {

template <typename T> struct DeltaOps;
template <> struct DeltaOps<bf16_t> {
    static constexpr int SL = 32, FE = 8, TPS = 2;      // contraction indices of a slab, elements of a fragment, result tiles that make a slab
    static constexpr int NLOW = 6;                      // fragments of a 64 x 64 lower (or upper) triangular operand
    typedef bf16x8 Frag;
    static __device__ __forceinline__ f32x4 mma(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ int row(int t, int m) { return 32 * (t >> 1) + 8 * (m >> 2) + 4 * (t & 1) + (m & 3); }
    static constexpr __device__ __forceinline__ bool low(int t, int s) { return s <= t >> 1; }
    static constexpr __device__ __forceinline__ int low_at(int t, int s) { return t < 2 ? t : 2 * (t - 1) + s; }              // t >= 2: slabs 0, 1
    static constexpr __device__ __forceinline__ bool up(int t, int s) { return s >= t >> 1; }
    static constexpr __device__ __forceinline__ int up_at(int t, int s) { return t < 2 ? 2 * t + s : 2 + t; }                 // t < 2: slabs 0, 1
};
template <> struct DeltaOps<float> {
    static constexpr int SL = 16, FE = 4, TPS = 1, NLOW = 10;
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
// four numbers as sums of NP bf16 numbers each, two to a register
template <int NP> struct DeltaSplit4 {
    uint2 p[NP];
    __device__ __forceinline__ explicit DeltaSplit4(const f32x4& v) {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        float r[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            unsigned w[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const f32x2 x = {r[2 * j], r[2 * j + 1]};
                w[j] = __builtin_bit_cast(unsigned, __builtin_convertvector(x, bf16x2));
                r[2 * j] -= __uint_as_float(w[j] << 16);
                r[2 * j + 1] -= __uint_as_float(w[j] & 0xffff0000u);
            }
            p[i] = uint2{w[0], w[1]};
        }
    }
};
// slab s of a column of result tiles, each value times f[...] of its tile and register, as a B operand
template <typename T, int NP> __device__ __forceinline__ void delta_pack(const f32x4* tile, int s, DeltaParts<T, NP>& o) {
    constexpr int FE = DeltaOps<T>::FE, TPS = DeltaOps<T>::TPS;
    float x[FE];
#pragma unroll
    for (int e = 0; e < FE; ++e) x[e] = tile[TPS * s + e / 4][e % 4];
    delta_split<T, NP>(x, o);
}
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

// Tiles of K and Q in LDS: rows of d elements without padding, the 16-byte pieces of a row permuted by an exclusive or with a number made of the row, so that
// neither a fragment along the row (sixteen rows' pieces of one column) nor, 16 bits, a transposing read (four rows, four pieces) meets itself on a bank.
template <typename T, int D> struct DeltaTile {
    static constexpr int ROWB = D * (int)sizeof(T), PPR = ROWB / 16, BYTES = 64 * ROWB;
    static __device__ __forceinline__ int turn(int row) {
        return sizeof(T) == 4 ? row & 15 : D == 128 ? ((row & 3) << 2) | ((row >> 3) & 3) : (((row >> 1) & 1) << 2) | ((row >> 3) & 3);
    }
    // bytes: the lane's place in the fragment (tile 0, slab 0) along the rows; slab s: xor 64 s; tile t: + tile_off(t)
    static __device__ __forceinline__ unsigned nat(int n, int g) {
        const int row = DeltaOps<T>::row(0, n);
        return row * ROWB + ((g ^ turn(row)) << 4);
    }
    static constexpr __device__ __forceinline__ unsigned tile_off(int t) { return sizeof(T) == 4 ? 16 * t * ROWB : (32 * (t >> 1) + 4 * (t & 1)) * ROWB; }
};

// The transposed tile as an A operand: rows of result tiles 2 tp, 2 tp + 1 (bf16) are the tile's columns, the contraction its 64 rows: fragments [tile % 2][slab] of
// one tp.  base: LDS address of the tile plus the lane's share tr(); xor 64 tp.
template <int D> __device__ __forceinline__ unsigned delta_tr(int lane) {
    const int g = lane >> 4, j = lane & 15, row = 8 * g + (j >> 2);
    return row * D * 2 + (((j & 3) ^ DeltaTile<bf16_t, D>::turn(row)) << 4);
}
template <int D> __device__ __forceinline__ void delta_ld_tr(unsigned at, bf16x8 (&f)[2][2]) {
    union U { unsigned long long v[2]; bf16x8 f; } u[4];
    constexpr int R4 = 4 * D * 2, R32 = 32 * D * 2;
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%9\n\tds_read_b64_tr_b16 %1, %8 offset:%10\n\t"
                 "ds_read_b64_tr_b16 %2, %8 offset:%11\n\tds_read_b64_tr_b16 %3, %8 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %4, %8 offset:%13\n\tds_read_b64_tr_b16 %5, %8 offset:%14\n\t"
                 "ds_read_b64_tr_b16 %6, %8 offset:%15\n\tds_read_b64_tr_b16 %7, %8 offset:%16\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(u[0].v[0]), "=&v"(u[0].v[1]), "=&v"(u[1].v[0]), "=&v"(u[1].v[1]), "=&v"(u[2].v[0]), "=&v"(u[2].v[1]), "=&v"(u[3].v[0]), "=&v"(u[3].v[1])
                 : "v"(at), "n"(0), "n"(R4), "n"(R32), "n"(R32 + R4), "n"(8), "n"(R4 + 8), "n"(R32 + 8), "n"(R32 + R4 + 8)
                 : "memory");
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int s = 0; s < 2; ++s) f[b][s] = u[2 * b + s].f;
}

}  // namespace path
