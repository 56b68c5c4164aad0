// Chunks of new tokens for a paged cache, bf16: the triangular transform of tiles of 64 tokens, the queries' way through the tiles
// to the chunk's start, and the keys' and the transitions' to its end.  (fp32, and what the quantities are: paged_chunk.hip.)
//
// Inputs are bf16 numbers and multiplied as they are.  What is computed from them -- T, T D, L, L T, Z, the carried keys, X and W X -- is
// multiplied as a sum of two bf16 numbers, hi + lo (17 bits; products hi hi + hi lo + lo hi): one fp16 number each
// leaves the log-sum-exp 2e-6 of itself off, through errors that all keys of a row share; so 1e-7, and with bf16's range.
// On the matrix units that is little: these products are a small part of the call, and a chain of short steps.
//
// The transform of a tile is a chain of nine small products and a substitution, 13 us with the launch for 8 tiles of 16 heads (16 with the queries' part,
// d = 128; in fp32 throughout 65): loads 5 us, the inverse 2, the rest 1 each.
#include <type_traits>

#include "paged_decl.h"

namespace path {

constexpr int C16_THREADS = 512, C16_LT = 72, C16_LF = 68;      // row lengths in LDS: 64 x 64 pairs, 64 x 64 fp32
template <int D> constexpr size_t chunk16_smem() { return (size_t)3 * 64 * (D + 8) * 2 + 2 * 64 * C16_LF * 4 + 4 * 2 * 64 * C16_LT * 2 + 64 * 4 + 256 * 4; }

struct Pair { bf16_t *hi, *lo; };
__device__ __forceinline__ void put_pair(const Pair& p, int i, float x) {
    const bf16_t h = (bf16_t)x;
    p.hi[i] = h;
    p.lo[i] = (bf16_t)(x - (float)h);
}
template <int K, bool TA, bool TB>
__device__ __forceinline__ void mm_pairs(f32x16& acc, const Pair& A, int lda, int ar, const Pair& B, int ldb, int br, int l32, int h) {
    mm<bf16_t, K, TA, TB>(acc, A.hi, lda, ar, B.hi, ldb, br, l32, h);
    mm<bf16_t, K, TA, TB>(acc, A.hi, lda, ar, B.lo, ldb, br, l32, h);
    mm<bf16_t, K, TA, TB>(acc, A.lo, lda, ar, B.hi, ldb, br, l32, h);
}

// One workgroup per tile and key head; 32 x 32 blocks by the eight waves, two 64 x 64 matrices at a time or one of d x 64.
template <int D>
__global__ __launch_bounds__(C16_THREADS, 1) void paged_chunk16_kernel(PagedArgs a) {
    constexpr int LD = D + 8, LT = C16_LT, LF = C16_LF, NT = C16_THREADS;
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    bf16_t* const W = reinterpret_cast<bf16_t*>(smem);
    bf16_t* const K = W + 64 * LD;
    bf16_t* const Q = K + 64 * LD;
    float* const F1 = reinterpret_cast<float*>(Q + 64 * LD);      // N; then, with F2, the pair L T
    float* const F2 = F1 + 64 * LF;                               // (I + N)^{-1}
    bf16_t* const pairs = reinterpret_cast<bf16_t*>(F2 + 64 * LF);
    const Pair Tp{pairs, pairs + 64 * LT}, Dt{pairs + 2 * 64 * LT, pairs + 3 * 64 * LT}, Lp{pairs + 4 * 64 * LT, pairs + 5 * 64 * LT},
        Ut{pairs + 6 * 64 * LT, pairs + 7 * 64 * LT}, LTp{reinterpret_cast<bf16_t*>(F1), reinterpret_cast<bf16_t*>(F1) + 64 * LT};
    static_assert(2 * 64 * LT * 2 <= 2 * 64 * LF * 4, "L T fits where N and its inverse were");
    float* const beta = reinterpret_cast<float*>(pairs + 8 * 64 * LT);
    float* const red = beta + 64;

    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hh = lane >> 5;
    const int tile = blockIdx.x % a.tiles, h = blockIdx.x / a.tiles, Hq = a.H * a.G;
    int s = 0;
    for (int i = 0; i < a.nseq; i += 64) s += __popcll(__ballot(i + lane < a.nseq && first_tile(a, min(i + lane, a.nseq - 1)) <= tile));
    s = __builtin_amdgcn_readfirstlane(max(0, s - 1));
    const PagedSeq q = paged_seq(a, s);
    const int c = tile - first_tile(a, s), m = q.m - 64 * c;
    if (q.m <= a.few_limit || c < 0 || m <= 0) return;
    const int tok0 = q.t0 + 64 * c;

    const bf16_t* const vg = reinterpret_cast<const bf16_t*>(a.v);
    auto stage = [&](bf16_t* dst, const void* src, int heads, int head) {
        const bf16_t* const p = reinterpret_cast<const bf16_t*>(src);
#pragma unroll
        for (int i0 = 0; i0 < 64 * D / 8; i0 += NT) {
            const int i = i0 + tid, t = i / (D / 8), e = (i % (D / 8)) * 8;
            u32x4 x = {0, 0, 0, 0};
            if (t < m) x = *reinterpret_cast<const u32x4*>(p + ((long long)(tok0 + t) * heads + head) * D + e);
            *reinterpret_cast<u32x4*>(dst + t * LD + e) = x;
        }
    };
    stage(W, a.w, a.H, h);
    stage(K, a.k, a.H, h);
    if (a.attn) stage(Q, a.q, Hq, h * a.G);
    if (tid < 64) beta[tid] = tid < m ? (float)reinterpret_cast<const bf16_t*>(a.beta)[(long long)(tok0 + tid) * a.H + h] : 0.f;
    if (a.cpages) {      // gate sums: c of the last cached token, the earlier tiles' gates, then one by one
        const bf16_t* const fg = reinterpret_cast<const bf16_t*>(a.log_f);
        if (tid < 256) {
            float x = 0.f;
            for (int t = tid; t < 64 * c; t += 256) x += (float)fg[(long long)(q.t0 + t) * a.H + h];
            red[tid] = x;
        }
        __syncthreads();
        if (wv == 0) {
            float y = red[lane] + red[64 + lane] + red[128 + lane] + red[192 + lane];
            for (int o = 32; o; o >>= 1) y += __shfl_xor(y, o);
            const long long r = q.n > 0 ? paged_row(a, s, h, q.n - 1) : -1;
            y += r >= 0 ? a.cpages[r] : 0.f;
            float z = lane < m ? (float)fg[(long long)(tok0 + lane) * a.H + h] : 0.f;
            for (int o = 1; o < 64; o <<= 1) { const float b = __shfl_up(z, o); if (lane >= o) z += b; }
            if (lane < m) a.crow[(long long)(tok0 + lane) * a.H + h] = y + z;
            if (a.append && lane < m) {
                const long long w = paged_row(a, s, h, q.n + 64 * c + lane);
                if (w >= 0) a.cpages[w] = y + z;
            }
        }
    }
    if (a.append)
        for (int i = tid; i < 64 * (D / 8); i += NT) {
            const int t = i / (D / 8), e = (i % (D / 8)) * 8;
            const long long r = t < m ? paged_row(a, s, h, q.n + 64 * c + t) : -1;
            if (r >= 0) *reinterpret_cast<u32x4*>(reinterpret_cast<bf16_t*>(a.vpages) + r * D + e) = *reinterpret_cast<const u32x4*>(vg + ((long long)(tok0 + t) * a.H + h) * D + e);
        }
    const size_t th = ((size_t)tile * a.H + h) * 64 * D;
    const size_t lo = (size_t)a.tiles * a.H * 64 * D;      // kt, zt: all hi tiles, then all lo tiles
    bf16_t* const kt = reinterpret_cast<bf16_t*>(a.kt) + th;
    bf16_t* const zt = reinterpret_cast<bf16_t*>(a.zt) + th;
    __syncthreads();

    const bool first = wv < 4;                            // which of two 64 x 64 matrices
    const int rb = (wv >> 1) & 1, cb = wv & 1;
    auto each = [&](const f32x16& v, auto f) {            // f(row, column, value) of this wave's block of a 64 x 64 matrix
#pragma unroll
        for (int j = 0; j < 16; ++j) f(32 * rb + acc_row(j, hh), 32 * cb + l32, v[j]);
    };
    auto lower = [&]() {                                  // L = lower(Q W^T)
        f32x16 v = zero16();
        mm<bf16_t, D, false, false>(v, Q, LD, 32 * rb, W, LD, 32 * cb, l32, hh);
        each(v, [&](int r, int k, float x) { put_pair(Lp, r * LT + k, k <= r ? x : 0.f); });
    };
    {   // N = diag(beta) strictLower(W W^T); D^T = strictUpper(K W^T)
        f32x16 v = zero16();
        mm<bf16_t, D, false, false>(v, first ? W : K, LD, 32 * rb, W, LD, 32 * cb, l32, hh);
        if (first) each(v, [&](int r, int k, float x) { F1[r * LF + k] = k < r ? beta[r] * x : 0.f; F2[r * LF + k] = 0.f; });
        else each(v, [&](int r, int k, float x) { put_pair(Dt, r * LT + k, k > r ? x : 0.f); });
    }
    __syncthreads();
    // (I + N)^{-1}: the 16 x 16 blocks on the diagonal by substitution, a column per thread
    if (wv == 0) {
        const int b = lane & ~15, j = lane & 15;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float y = i == j ? 1.f : 0.f;
#pragma unroll
            for (int t = 0; t < i; ++t) y -= F1[(b + i) * LF + b + t] * x[t];
            x[i] = y;
            F2[(b + i) * LF + b + j] = y;
        }
    } else if (!first && a.attn) lower();
    __syncthreads();
    // ... then twice the lower left quarter, -T22 (N21 T11), by 16 x 16 blocks; a product's result is the next one's right operand as it stands
    const int g = lane >> 4, c16 = lane & 15;
    auto quarter = [&](auto half, int b, int rq, int cq) {
        constexpr int HB = decltype(half)::value, NB = HB / 16;
        f32x4 tmp[NB];
#pragma unroll
        for (int r = 0; r < NB; ++r) {
            tmp[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < HB; k += 4)
                tmp[r] = __builtin_amdgcn_mfma_f32_16x16x4f32(F1[(b + HB + 16 * r + c16) * LF + b + k + g], F2[(b + k + g) * LF + b + 16 * cq + c16], tmp[r], 0, 0, 0);
        }
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < NB; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                y = __builtin_amdgcn_mfma_f32_16x16x4f32(F2[(b + HB + 16 * rq + c16) * LF + b + HB + 16 * r + 4 * g + i], tmp[r][i], y, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) F2[(b + HB + 16 * rq + 4 * g + i) * LF + b + 16 * cq + c16] = -y[i];
    };
    if (wv < 2) quarter(std::integral_constant<int, 16>(), 32 * wv, 0, 0);
    __syncthreads();
    if (wv < 4) quarter(std::integral_constant<int, 32>(), 0, wv >> 1, wv & 1);
    __syncthreads();
    for (int i = tid; i < 64 * 64; i += NT) put_pair(Tp, (i >> 6) * LT + (i & 63), F2[(i >> 6) * LF + (i & 63)] * beta[i & 63]);      // T
    __syncthreads();
    if (first) {   // (T D)^T
        f32x16 v = zero16();
        mm_pairs<64, false, false>(v, Dt, LT, 32 * rb, Tp, LT, 32 * cb, l32, hh);
        each(v, [&](int r, int k, float x) { put_pair(Ut, r * LT + k, x); });
    }
    auto product = [&](int b, const Pair& B) {      // block b of B W: rows 32 (b % 2), d 32 (b / 2)
        f32x16 v = zero16();
        mm<bf16_t, 64, false, true>(v, B.hi, LT, 32 * (b & 1), W, LD, 32 * (b >> 1), l32, hh);
        mm<bf16_t, 64, false, true>(v, B.lo, LT, 32 * (b & 1), W, LD, 32 * (b >> 1), l32, hh);
        return v;
    };
    // A block as a pair to memory: neighbouring lanes exchange, so that each has two columns of one of two rows, and 64 bytes of a row go out in one piece.
    // (Four rows' eight bytes per lane, the transposed product, went out in pieces of sixteen: the stores took 4 us more of a tile's 17.)
    auto store_pair = [&](bf16_t* p, int b, const f32x16& v) {
        const bool even = !(lane & 1);
        typedef bf16_t V2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
            const float got = __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(even ? v[j + 1] : v[j]), 0xb1, 0xf, 0xf, true));
            const float x0 = even ? v[j] : got, x1 = even ? got : v[j + 1];
            bf16_t* const at = p + (32 * (b & 1) + acc_row(j, hh) + (even ? 0 : 1)) * D + 32 * (b >> 1) + (l32 & ~1);
            V2 x, y;
            x[0] = (bf16_t)x0;
            x[1] = (bf16_t)x1;
            y[0] = (bf16_t)(x0 - (float)x[0]);
            y[1] = (bf16_t)(x1 - (float)x[1]);
            *reinterpret_cast<V2*>(at) = x;
            *reinterpret_cast<V2*>(at + lo) = y;
        }
    };
    auto less = [&](const bf16_t* M, int b, f32x16 v) {      // the block of M - v
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = (float)M[(32 * (b & 1) + acc_row(j, hh)) * LD + 32 * (b >> 1) + l32] - v[j];
        return v;
    };
    if (!first)      // -Z = -T W
        for (int b = wv - 4; b < D / 16; b += 4) store_pair(zt, b, -product(b, Tp));
    __syncthreads();
    for (int b = wv; b < D / 16; b += 8) store_pair(kt, b, less(K, b, product(b, Ut)));      // carried keys K - (T D)^T W
    if (!a.attn) return;
    for (int gq = 0; gq < a.G; ++gq) {
        const int hq = h * a.G + gq;
        if (gq > 0) {
            __syncthreads();
            stage(Q, a.q, Hq, hq);
            __syncthreads();
            if (first) lower();
            __syncthreads();
        }
        if (first) {      // logits: Q K^T - L (T D)
            f32x16 v = zero16(), u = zero16();
            mm<bf16_t, D, false, false>(v, Q, LD, 32 * rb, K, LD, 32 * cb, l32, hh);
            mm_pairs<64, false, false>(u, Lp, LT, 32 * rb, Ut, LT, 32 * cb, l32, hh);
            float* const sd = a.sd + ((size_t)tile * Hq + hq) * 4096;
            each(v - u, [&](int r, int k, float x) { sd[r * 64 + k] = x; });
        } else {          // L T
            f32x16 v = zero16();
            mm_pairs<64, false, true>(v, Lp, LT, 32 * rb, Tp, LT, 32 * cb, l32, hh);
            each(v, [&](int r, int k, float x) { put_pair(LTp, r * LT + k, x); });
        }
        __syncthreads();
        for (int b = wv; b < D / 16; b += 8) {      // X = Q - (L T) W
            const f32x16 v = less(Q, b, product(b, LTp));
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int t = 32 * (b & 1) + acc_row(j, hh);
                if (t < m) a.x[((long long)(tok0 + t) * Hq + hq) * D + 32 * (b >> 1) + l32] = v[j];
            }
        }
    }
}

// ---- the way through the tiles ----
//
// 32 or 64 rows per workgroup, and four waves for each 16 of them, which share a step's work:
//     waves a   S = kt X^T (32 of the tile's 64 tokens each), softmax, O^T += V^T P^T: two online softmaxes, joined at the end.  scan: S are rows of keys, stored
//     waves b   Y = W X^T (32 tokens each), exchanged; X^T -= Z^T Y (half of d each), and X as operands to LDS for the next step
// The tile's operands come to LDS in two sets, each while the other is worked on: carried keys (hi, lo) and W; -Z (hi, lo) and V.
// Bound by the chain of steps, with 64 rows about 3 us each at d = 128 and 1.8 at 64: products of 1.0 us a SIMD, LDS of 0.9, 0.7 of waiting for the copies, and between
// them the latency of reads, packing and two barriers.  Per workgroup up to 144 KB of LDS, so one on a CU.  One wave for all of a row's work took 4.2 us a step, two
// 3.3; whole tiles from L2 to registers, without LDS, 7.5.
// The first workgroups are those of the append's scan, whose way is the longest: rows of the identity, of which S are rows of the
// keys carried to the chunk's end, and what is left of X the rows of H_{m-1} .. H_0.
// As an operand a lane holds elements 32 s + 4 g + 0..3 and 16 further on, as results have them; two eight-byte reads of the keys and of W, which like the
// transposing reads take whole sixteen-byte pieces off the banks (eight elements in a row cost the latter twice their time).
template <int D, int RS> constexpr size_t sweep16_smem() { return (size_t)6 * 64 * D * 2 + (size_t)RS * (D / 32) * 2 * 64 * 16 + RS * 2 * 2 * 64 * 16; }

// Place of an element in a tile of 64 rows: sixteen-byte pieces of a row exchanged by its turn, such that 32 lanes' eight bytes fall on all banks
// once, both of one piece's two halves in 16 rows (fragments along the row) and of 32 bytes in 8 rows (transposing reads).
template <int W> struct Turned16 {
    static __host__ __device__ __forceinline__ int turn(int row) {
        return W == 128 ? ((row & 3) << 2) | (((row >> 2) & 1) << 1) | ((row >> 3) & 1) : (((row >> 1) & 3) << 1) | ((row >> 3) & 1);
    }
    static __host__ __device__ __forceinline__ int at(int row, int col) { return row * W + ((((col >> 3) ^ turn(row)) << 3) | (col & 7)); }
};
// Fragments of two blocks of 16 rows: eight bytes at a and at b each; of a tile and of the one behind it, or of one.  (Left to the compiler these become
// reads of two rows at once, which take four times as long.)
template <int OFF, int ROWB>
__device__ __forceinline__ void rows_pair(unsigned a, unsigned b, bf16x8 (&f)[2], bf16x8 (&l)[2]) {
    constexpr int T = 64 * ROWB;
    union U { unsigned long long v[2]; bf16x8 f; } u[4];
    asm volatile("ds_read_b64 %0, %8 offset:%10\n\tds_read_b64 %1, %9 offset:%10\n\tds_read_b64 %2, %8 offset:%11\n\tds_read_b64 %3, %9 offset:%11\n\t"
                 "ds_read_b64 %4, %8 offset:%12\n\tds_read_b64 %5, %9 offset:%12\n\tds_read_b64 %6, %8 offset:%13\n\tds_read_b64 %7, %9 offset:%13\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(u[0].v[0]), "=&v"(u[0].v[1]), "=&v"(u[1].v[0]), "=&v"(u[1].v[1]), "=&v"(u[2].v[0]), "=&v"(u[2].v[1]), "=&v"(u[3].v[0]), "=&v"(u[3].v[1])
                 : "v"(a), "v"(b), "n"(OFF), "n"(OFF + 16 * ROWB), "n"(OFF + T), "n"(OFF + T + 16 * ROWB) : "memory");
    f[0] = u[0].f;
    f[1] = u[1].f;
    l[0] = u[2].f;
    l[1] = u[3].f;
}
template <int OFF, int ROWB>
__device__ __forceinline__ void rows_one(unsigned a, unsigned b, bf16x8 (&f)[2]) {
    union U { unsigned long long v[2]; bf16x8 f; } u[2];
    asm volatile("ds_read_b64 %0, %4 offset:%6\n\tds_read_b64 %1, %5 offset:%6\n\tds_read_b64 %2, %4 offset:%7\n\tds_read_b64 %3, %5 offset:%7\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(u[0].v[0]), "=&v"(u[0].v[1]), "=&v"(u[1].v[0]), "=&v"(u[1].v[1])
                 : "v"(a), "v"(b), "n"(OFF), "n"(OFF + 16 * ROWB) : "memory");
    f[0] = u[0].f;
    f[1] = u[1].f;
}
// Fragments (16 d x 32 tokens) of a tile's transpose for four blocks of 16 d, whose addresses are a0 .. a3: reads of rows 32 u + 4 g + 0..3 and
// of those 16 further on.  The waits are in the block.
template <int OFF, int ROWB>
__device__ __forceinline__ void turned_tr(unsigned a0, unsigned a1, unsigned a2, unsigned a3, bf16x8 (&f)[4]) {
    union U { unsigned long long v[2]; bf16x8 f; } u[4];
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %2, %9 offset:%12\n\tds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %4, %10 offset:%12\n\tds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %6, %11 offset:%12\n\tds_read_b64_tr_b16 %7, %11 offset:%13\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(u[0].v[0]), "=&v"(u[0].v[1]), "=&v"(u[1].v[0]), "=&v"(u[1].v[1]), "=&v"(u[2].v[0]), "=&v"(u[2].v[1]), "=&v"(u[3].v[0]), "=&v"(u[3].v[1])
                 : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "n"(OFF), "n"(OFF + 16 * ROWB) : "memory");
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = u[k].f;
}
// The same of a pair of tiles, one behind the other.
template <int OFF, int ROWB>
__device__ __forceinline__ void turned_tr_pair(unsigned a0, unsigned a1, unsigned a2, unsigned a3, bf16x8 (&f)[4], bf16x8 (&l)[4]) {
    constexpr int T = 64 * ROWB;
    union U { unsigned long long v[2]; bf16x8 f; } u[8];
    asm volatile("ds_read_b64_tr_b16 %0, %16 offset:%20\n\tds_read_b64_tr_b16 %1, %16 offset:%21\n\t"
                 "ds_read_b64_tr_b16 %2, %17 offset:%20\n\tds_read_b64_tr_b16 %3, %17 offset:%21\n\t"
                 "ds_read_b64_tr_b16 %4, %18 offset:%20\n\tds_read_b64_tr_b16 %5, %18 offset:%21\n\t"
                 "ds_read_b64_tr_b16 %6, %19 offset:%20\n\tds_read_b64_tr_b16 %7, %19 offset:%21\n\t"
                 "ds_read_b64_tr_b16 %8, %16 offset:%22\n\tds_read_b64_tr_b16 %9, %16 offset:%23\n\t"
                 "ds_read_b64_tr_b16 %10, %17 offset:%22\n\tds_read_b64_tr_b16 %11, %17 offset:%23\n\t"
                 "ds_read_b64_tr_b16 %12, %18 offset:%22\n\tds_read_b64_tr_b16 %13, %18 offset:%23\n\t"
                 "ds_read_b64_tr_b16 %14, %19 offset:%22\n\tds_read_b64_tr_b16 %15, %19 offset:%23\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(u[0].v[0]), "=&v"(u[0].v[1]), "=&v"(u[1].v[0]), "=&v"(u[1].v[1]), "=&v"(u[2].v[0]), "=&v"(u[2].v[1]), "=&v"(u[3].v[0]), "=&v"(u[3].v[1]),
                   "=&v"(u[4].v[0]), "=&v"(u[4].v[1]), "=&v"(u[5].v[0]), "=&v"(u[5].v[1]), "=&v"(u[6].v[0]), "=&v"(u[6].v[1]), "=&v"(u[7].v[0]), "=&v"(u[7].v[1])
                 : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "n"(OFF), "n"(OFF + 16 * ROWB), "n"(OFF + T), "n"(OFF + T + 16 * ROWB) : "memory");
#pragma unroll
    for (int k = 0; k < 4; ++k) { f[k] = u[k].f; l[k] = u[4 + k].f; }
}
// Results (16 (2 s + j / 4) + 4 g + j % 4 in place j of slab s) as operands
template <int N> __device__ __forceinline__ void pack_pairs(const f32x4* x, bf16x8* hi, bf16x8* lo) {
#pragma unroll
    for (int s = 0; s < N; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float v = x[2 * s + (j >> 2)][j & 3];
            hi[s][j] = (bf16_t)v;
            lo[s][j] = (bf16_t)(v - (float)hi[s][j]);
        }
}
__device__ __forceinline__ f32x4 mfma32(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

template <int D, bool SCAN, int RS>
__device__ __forceinline__ void sweep16(const PagedArgs& a, unsigned char* smem, int s, int h, int hq, int ct, int r0) {
    typedef Turned16<D> L;
    constexpr int ROWB = D * 2, TILE = 64 * ROWB, DT = D / 16, DS = D / 32, HT = DT / 2, HS = DS / 2, PPR = D / 8, RPI = 64 / PPR;
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15, Hq = a.H * a.G;
    const int rw = wv & (RS - 1), part = (wv / RS) & 1;      // its 16 rows, and which half of the work on them
    const bool carries = wv >= 2 * RS;                       // waves b
    const PagedSeq q = paged_seq(a, s);
    const int first = first_tile(a, s), row = r0 + 16 * rw + c;
    const int tok = SCAN ? 0 : q.t0 + 64 * ct + row;
    const bool there = SCAN || 64 * ct + row < q.m;
    const long long at = (long long)tok * Hq + hq;
    const size_t lo = (size_t)a.tiles * a.H * 64 * D;
    const bf16_t* const kt = reinterpret_cast<const bf16_t*>(a.kt);
    const bf16_t* const zt = reinterpret_cast<const bf16_t*>(a.zt);
    bf16x8* const sx = reinterpret_cast<bf16x8*>(smem + 6 * TILE) + rw * DS * 2 * 64 + lane;                            // X of the 16 rows: [slab][hi, lo][lane]
    bf16x8* const sy = reinterpret_cast<bf16x8*>(smem + 6 * TILE + RS * DS * 2 * 64 * 16) + rw * 2 * 2 * 64 + lane;      // Y: the same, two slabs

    // copies: the waves share a tile's rows, a row's pieces exchanged by its turn; rows of w and v past the last token: that token's
    auto copy = [&](int slot, const bf16_t* src, long long stride, int last) {
#pragma unroll
        for (int i0 = 0; i0 < 64 / RPI; i0 += 4 * RS) {
            const int i = i0 + wv, r = RPI * i + lane / PPR;
            if (i < 64 / RPI) {
                const bf16_t* const p = src + min(r, last) * stride + ((lane % PPR) ^ L::turn(r)) * 8;
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                                 (__attribute__((address_space(3))) void*)(smem + slot * TILE + RPI * i * ROWB), 16, 0, 0);
            }
        }
    };
    auto tile_at = [&](int j) { return ((size_t)(first + j) * a.H + h) * 64 * D; };
    auto user = [&](const void* p, int j) { return reinterpret_cast<const bf16_t*>(p) + ((long long)(q.t0 + 64 * j) * a.H + h) * D; };
    auto bring0 = [&](int j) {
        copy(0, kt + tile_at(j), D, 63);
        copy(1, kt + lo + tile_at(j), D, 63);
        copy(2, user(a.w, j), (long long)a.H * D, q.m - 64 * j - 1);
    };
    auto bring1 = [&](int j) {
        copy(3, zt + tile_at(j), D, 63);
        copy(4, zt + lo + tile_at(j), D, 63);
        if (!SCAN) copy(5, user(a.v, j), (long long)a.H * D, q.m - 64 * j - 1);
    };
    if (!SCAN) copy(5, user(a.v, ct), (long long)a.H * D, q.m - 64 * ct - 1);
    else bring1(ct - 1);
    if (ct > 0) bring0(ct - 1);

    const unsigned base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const unsigned tr = base + 3 * TILE + L::at(4 * g + (c >> 2), 4 * (c & 3)) * 2;      // of set 1; d block t: exclusive or 32 t
    const unsigned nat = base + part * 32 * ROWB + L::at(c, 4 * g) * 2;                  // of set 0, its 32 tokens; d slab s: exclusive or 64 s, its second half + 32
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};

    if (!carries) {
        f32x4 O[SCAN ? 1 : DT], S[2];
        float m_run = -INFINITY, l_run = 0.f, cq = 0.f;
        const float sl2 = a.scale * LOG2E;
        bf16x8 P;
        auto softmax = [&](int j, bool own) {
            float top = -INFINITY, ck[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) ck[i] = 0.f;
            if (a.cpages) {
#pragma unroll
                for (int i = 0; i < 8; ++i) ck[i] = a.crow[(long long)min(q.t0 + 64 * j + 32 * part + 16 * (i >> 2) + 4 * g + (i & 3), a.T - 1) * a.H + h];
            }
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float y = S[b][i] * sl2 + (cq - ck[4 * b + i]) * LOG2E;      // (no gates: both are zero)
                    if (own) y = 32 * part + 16 * b + 4 * g + i <= row ? y : -INFINITY;
                    S[b][i] = y;
                    top = fmaxf(top, y);
                }
            const float now = fmaxf(m_run, max_rows(top)), ref = now == -INFINITY ? 0.f : now, f = __builtin_amdgcn_exp2f(m_run - ref);
            m_run = now;
            float sum = 0.f;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) { S[b][i] = __builtin_amdgcn_exp2f(S[b][i] - ref); sum += S[b][i]; }
            l_run = l_run * f + sum;
#pragma unroll
            for (int t = 0; t < DT; ++t) O[t] *= f;
#pragma unroll
            for (int k = 0; k < 8; ++k) P[k] = (bf16_t)S[k >> 2][k & 3];
        };
        auto values = [&]() {
            const unsigned v0 = tr + part * 32 * ROWB;
#pragma unroll
            for (int t = 0; t < DT; t += 4) {      // four blocks at a time, none waiting for its own last product
                bf16x8 v[4];
                turned_tr<2 * TILE, ROWB>(v0 ^ (32 * t), v0 ^ (32 * t + 32), v0 ^ (32 * t + 64), v0 ^ (32 * t + 96), v);
#pragma unroll
                for (int k = 0; k < 4; ++k) O[t + k] = mfma32(v[k], P, O[t + k]);
            }
        };
        // The own tile's values again, each row with no token behind it: what a later one holds would show in the product with its weight 0 if it is an infinity or
        // NaN.  Then this takes the product's place (and where a row's own are such: it gives what the product gave).
        auto own_values = [&]() {
#pragma unroll
            for (int t = 0; t < DT; ++t) O[t] = zero;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                for (int from = 0; from < 4; ++from) {
                    const int key = 32 * part + 16 * (k >> 2) + 4 * from + (k & 3);
                    const float p = __shfl((float)P[k], 16 * from + c);
                    if (!there || key > row) continue;
                    const bf16_t* const v = user(a.v, ct) + (long long)key * a.H * D + 4 * g;
#pragma unroll
                    for (int t = 0; t < DT; ++t) {
                        const bf16x4 x = *reinterpret_cast<const bf16x4*>(v + 16 * t);
#pragma unroll
                        for (int i = 0; i < 4; ++i) O[t][i] += p * (float)x[i];
                    }
                }
        };
        long long place[2];      // SCAN: where this lane's key of each block goes
        auto places = [&](int j) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int t = 64 * j + 32 * part + 16 * b + c;
                place[b] = t < q.m ? paged_row(a, s, h, q.n + t) : -1;
            }
        };
        if constexpr (SCAN) {
            places(ct - 1);
            wait_async_and_sync();
            lds_barrier();
        } else {      // the tile's own logits are there
#pragma unroll
            for (int t = 0; t < DT; ++t) O[t] = zero;
            if (a.cpages && there) cq = a.crow[(long long)tok * a.H + h];
            const float* const sd = a.sd + ((size_t)(first + ct) * Hq + hq) * 4096 + row * 64 + 32 * part;
#pragma unroll
            for (int b = 0; b < 2; ++b) S[b] = *reinterpret_cast<const f32x4*>(sd + 16 * b + 4 * g);
            softmax(ct, true);
            wait_async_and_sync();
            values();
            if (__any(not_finite<DT>(O))) own_values();
            lds_barrier();
            if (ct > 0) bring1(ct - 1);
        }
        for (int j = ct - 1; j >= 0; --j) {
            // set 0 and X are there
            f32x4 R[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) S[b] = R[b] = zero;
#pragma unroll
            for (int sl = 0; sl < DS; ++sl) {
                const bf16x8 xh = sx[(2 * sl) * 64], xl = sx[(2 * sl + 1) * 64];
                bf16x8 kh[2], kl[2];
                rows_pair<0, ROWB>(nat ^ (64 * sl), nat ^ (64 * sl + 32), kh, kl);
                // (scan: transposed, a lane has four consecutive elements of a key)
#pragma unroll
                for (int b = 0; b < 2; ++b) S[b] = SCAN ? mfma32(xh, kh[b], S[b]) : mfma32(kh[b], xh, S[b]);
#pragma unroll
                for (int b = 0; b < 2; ++b) R[b] = SCAN ? mfma32(xl, kh[b], R[b]) : mfma32(kh[b], xl, R[b]);
#pragma unroll
                for (int b = 0; b < 2; ++b) S[b] = SCAN ? mfma32(xh, kl[b], S[b]) : mfma32(kl[b], xh, S[b]);
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) S[b] += R[b];
            wait_async_and_sync();      // set 1 is there, set 0 and X are free
            if (j > 0) bring0(j - 1);
            if constexpr (SCAN) {
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    bf16x4 v;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = (bf16_t)S[b][i];
                    if (place[b] >= 0) *reinterpret_cast<bf16x4*>(reinterpret_cast<bf16_t*>(a.kpages) + place[b] * D + r0 + 16 * rw + 4 * g) = v;
                }
                if (j > 0) places(j - 1);
            } else {
                softmax(j, false);
                values();
            }
            wait_async_and_sync();      // set 0 and X are there, set 1 is free
            if (j > 0) bring1(j - 1);
        }
        if constexpr (!SCAN) {      // the two halves' softmaxes joined, where set 0 was
            l_run = sum_rows(l_run);
            float* const p = reinterpret_cast<float*>(smem) + rw * (DT * 256 + 128);
            if (part == 1) {
#pragma unroll
                for (int t = 0; t < DT; ++t) *reinterpret_cast<f32x4*>(p + t * 256 + lane * 4) = O[t];
                p[DT * 256 + lane] = m_run;
                p[DT * 256 + 64 + lane] = l_run;
            }
            lds_barrier();
            if (part == 0 && there) {
                const float m2 = p[DT * 256 + lane], now = fmaxf(m_run, m2), f1 = __builtin_amdgcn_exp2f(m_run - now), f2 = __builtin_amdgcn_exp2f(m2 - now);      // (the own tile's first half has the row's first keys: now is finite)
                l_run = l_run * f1 + p[DT * 256 + 64 + lane] * f2;
#pragma unroll
                for (int t = 0; t < DT; ++t) O[t] = O[t] * f1 + *reinterpret_cast<const f32x4*>(p + t * 256 + lane * 4) * f2;
                if (q.n == 0) {      // nothing cached: that was all
                    const float inv = 1.f / l_run;
#pragma unroll
                    for (int t = 0; t < DT; ++t) {
                        bf16x4 v;
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = (bf16_t)(O[t][i] * inv);
                        *reinterpret_cast<bf16x4*>(reinterpret_cast<bf16_t*>(a.o) + at * D + 16 * t + 4 * g) = v;
                    }
                    if (g == 0) a.lse[at] = (now + __builtin_amdgcn_logf(l_run)) * LN2;
                } else {
#pragma unroll
                    for (int t = 0; t < DT; ++t) *reinterpret_cast<f32x4*>(a.many_o + at * D + 16 * t + 4 * g) = O[t];
                    if (g == 0) { a.many_ml[2 * at] = now; a.many_ml[2 * at + 1] = l_run; }
                }
            }
        }
    } else {
        f32x4 x[HT], Y[2];      // its half of X
#pragma unroll
        for (int t = 0; t < HT; ++t) {
            const int d = 16 * (HT * part + t) + 4 * g;
            x[t] = zero;
            if constexpr (SCAN) {
#pragma unroll
                for (int i = 0; i < 4; ++i) x[t][i] = d + i == row ? 1.f : 0.f;
            } else if (there) {
                x[t] = *reinterpret_cast<const f32x4*>(a.x + at * D + d);
            }
        }
        auto hand_over = [&]() {
            bf16x8 xh[HS], xl[HS];
            pack_pairs<HS>(x, xh, xl);
#pragma unroll
            for (int sl = 0; sl < HS; ++sl) { sx[(2 * (HS * part + sl)) * 64] = xh[sl]; sx[(2 * (HS * part + sl) + 1) * 64] = xl[sl]; }
        };
        if (ct > 0) hand_over();
        wait_async_and_sync();
        lds_barrier();
        if (!SCAN && ct > 0) bring1(ct - 1);
        for (int j = ct - 1; j >= 0; --j) {
            bf16x8 xh[DS], xl[DS];
#pragma unroll
            for (int sl = 0; sl < DS; ++sl) { xh[sl] = sx[(2 * sl) * 64]; xl[sl] = sx[(2 * sl + 1) * 64]; }
            f32x4 R[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) Y[b] = R[b] = zero;
#pragma unroll
            for (int sl = 0; sl < DS; ++sl) {
                bf16x8 w[2];
                rows_one<2 * TILE, ROWB>(nat ^ (64 * sl), nat ^ (64 * sl + 32), w);
#pragma unroll
                for (int b = 0; b < 2; ++b) Y[b] = mfma32(w[b], xh[sl], Y[b]);
#pragma unroll
                for (int b = 0; b < 2; ++b) R[b] = mfma32(w[b], xl[sl], R[b]);
            }
            bf16x8 yh[2], yl[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) Y[b] += R[b];
            pack_pairs<1>(Y, yh, yl);
            sy[(2 * part) * 64] = yh[0];
            sy[(2 * part + 1) * 64] = yl[0];
            wait_async_and_sync();
            if (j > 0) bring0(j - 1);
#pragma unroll
            for (int u = 0; u < 2; ++u) { yh[u] = sy[(2 * u) * 64]; yl[u] = sy[(2 * u + 1) * 64]; }
            const unsigned z0 = tr ^ (32 * HT * part);
            bf16x8 zh[4], zl[4];
            if constexpr (HT == 4) {
                turned_tr_pair<0, ROWB>(z0, z0 ^ 32, z0 ^ 64, z0 ^ 96, zh, zl);
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = mfma32(zh[k], yh[0], x[k]);
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = mfma32(zh[k], yl[0], x[k]);
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = mfma32(zl[k], yh[0], x[k]);
                turned_tr_pair<32 * ROWB, ROWB>(z0, z0 ^ 32, z0 ^ 64, z0 ^ 96, zh, zl);
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = mfma32(zh[k], yh[1], x[k]);
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = mfma32(zh[k], yl[1], x[k]);
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = mfma32(zl[k], yh[1], x[k]);
            } else {      // two blocks, both slabs
                turned_tr_pair<0, ROWB>(z0, z0 ^ 32, z0 + 32 * ROWB, (z0 ^ 32) + 32 * ROWB, zh, zl);
                f32x4 y[2] = {zero, zero};
#pragma unroll
                for (int k = 0; k < 4; ++k) { f32x4& v = k < 2 ? x[k] : y[k - 2]; v = mfma32(zh[k], yh[k >> 1], v); }
#pragma unroll
                for (int k = 0; k < 4; ++k) { f32x4& v = k < 2 ? x[k] : y[k - 2]; v = mfma32(zh[k], yl[k >> 1], v); }
#pragma unroll
                for (int k = 0; k < 4; ++k) { f32x4& v = k < 2 ? x[k] : y[k - 2]; v = mfma32(zl[k], yh[k >> 1], v); }
#pragma unroll
                for (int k = 0; k < 2; ++k) x[k] += y[k];
            }
            if (j > 0) hand_over();
            wait_async_and_sync();
            if (j > 0) bring1(j - 1);
        }
        if constexpr (SCAN) {
            half_t* const p = reinterpret_cast<half_t*>(a.pt) + (((size_t)s * a.H + h) * D + row) * D;
#pragma unroll
            for (int t = 0; t < HT; ++t) {
                const int d = 16 * (HT * part + t) + 4 * g;
                halfx4 v;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = (half_t)(x[t][i] - (d + i == row ? 1.f : 0.f));
                *reinterpret_cast<halfx4*>(p + d) = v;
            }
        } else {
            if (there && q.n > 0) {
#pragma unroll
                for (int t = 0; t < HT; ++t) *reinterpret_cast<f32x4*>(a.x + at * D + 16 * (HT * part + t) + 4 * g) = x[t];
            }
            lds_barrier();      // (where waves a join their halves)
        }
    }
}

template <int D, int RS>
__global__ __launch_bounds__(256 * RS, 1) void paged_sweep16_kernel(PagedArgs a) {
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    constexpr int BLOCKS = D / (16 * RS), HALVES = 4 / RS;      // workgroups for the identity's rows, for a tile's
    const int lane = threadIdx.x & 63, Hq = a.H * a.G, scans = a.append ? a.nseq * a.H * BLOCKS : 0;
    int x = blockIdx.x;
    if (x < scans) {
        const int r0 = 16 * RS * (x % BLOCKS); x /= BLOCKS;
        const int s = x / a.H, m = paged_seq(a, s).m;
        if (m <= a.few_limit) return;
        sweep16<D, true, RS>(a, smem, s, x % a.H, 0, (m + 63) >> 6, r0);
        return;
    }
    x -= scans;
    const int hq = x % Hq; x /= Hq;
    const int tile = a.tiles - 1 - x / HALVES, r0 = 16 * RS * (x % HALVES);      // (the last tiles have the longest way)
    int s = 0;
    for (int i = 0; i < a.nseq; i += 64) s += __popcll(__ballot(i + lane < a.nseq && first_tile(a, min(i + lane, a.nseq - 1)) <= tile));
    s = __builtin_amdgcn_readfirstlane(max(0, s - 1));
    const int m = paged_seq(a, s).m, ct = tile - first_tile(a, s);
    if (m <= a.few_limit || ct < 0 || 64 * ct + r0 >= m) return;
    sweep16<D, false, RS>(a, smem, s, hq / a.G, hq, __builtin_amdgcn_readfirstlane(ct), r0);
}

template <int D>
static hipError_t launch_chunk16_t(const PagedArgs& a, hipStream_t st) {
    constexpr size_t bytes = chunk16_smem<D>();
    static_assert(bytes <= 160 * 1024, "LDS");
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_chunk16_kernel<D>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL((paged_chunk16_kernel<D>), dim3((unsigned)(a.tiles * a.H)), dim3(C16_THREADS), bytes, st, a);
    return hipGetLastError();
}
hipError_t launch_paged_chunk16(const PagedArgs& a, int d, hipStream_t st) { return d == 64 ? launch_chunk16_t<64>(a, st) : launch_chunk16_t<128>(a, st); }
template <int D, int RS>
static hipError_t launch_sweep16_t(const PagedArgs& a, hipStream_t st) {
    constexpr size_t bytes = sweep16_smem<D, RS>();
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_sweep16_kernel<D, RS>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (attr != hipSuccess) return attr;
    const unsigned grid = (unsigned)((a.append ? a.nseq * a.H * (D / (16 * RS)) : 0) + (a.attn ? a.tiles * a.H * a.G * (4 / RS) : 0));
    hipLaunchKernelGGL((paged_sweep16_kernel<D, RS>), dim3(grid), dim3(256 * RS), bytes, st, a);
    return hipGetLastError();
}
// 32 rows per workgroup shorten a step (two waves a SIMD instead of four), 64 bring the tiles for twice as many rows.  A CU holds one workgroup, and those with the
// longest ways start first, so that 32 rows, two workgroups for every tile and head, win up to about two for each CU: the last tiles' fill the chip, the first ones' short
// ways run behind them.  us a call over nothing, 32 / 64 rows, 16 heads, d = 128: 512 tokens 36.0 / 40.4, 1000 (256 tiles and heads) 56.2 / 61.2, 1080 (272) 72.8 / 74.3,
// 1150 (288) 78.6 / 77.3, 1500 (384) 111 / 93.5; with the append, whose scan's workgroups come on top, 1000 66.7 / 67.4, 1080 84.7 / 81.5; d = 64: 1080 48.8 / 50.9, 1300
// 54.7 / 56.2, 1500 61.8 / 60.4.  The append alone, 512 tokens, d = 128: 32 heads 53.5 / 59.1, 64 (8192) 72.2 / 69.5, 96 102 / 83.7; d = 64: 8192 64.7 / 66.0.
hipError_t launch_paged_sweep16(const PagedArgs& a, int d, hipStream_t st) {
    const bool narrow = a.attn ? (a.T / 64 + 1) * a.H * a.G <= 272 : a.nseq * a.H * d <= 8192;
    if (narrow) return d == 64 ? launch_sweep16_t<64, 2>(a, st) : launch_sweep16_t<128, 2>(a, st);
    return d == 64 ? launch_sweep16_t<64, 4>(a, st) : launch_sweep16_t<128, 4>(a, st);
}

}  // namespace path
