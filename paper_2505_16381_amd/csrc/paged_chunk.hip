// Chunks of new tokens for a paged cache, fp32: the triangular transform of tiles of 64 tokens, the queries' way through the tiles to
// the chunk's start, and the keys' and the transitions' to its end.  (bf16: paged_chunk16.hip.)
//
// Per tile and key head (paged_chunk_kernel), with the matrices of paged_decl.h restricted to the tile's tokens:
//     kt  K - (T D)^T W       keys carried to the tile's right edge
//     wt, zt, vt              W, -Z^T and V^T: of the tile's product I - W^T Z only the two factors are kept, as a product with 64 rows costs
//                             what one with the d x d matrix costs at d = 128
//     x   Q - (L T) W         queries as they stand at the tile's left edge
//     sd  Q K^T - L (T D)     logits inside the tile
//
// paged_sweep_kernel carries rows X through earlier tiles, right to left: S = kt X^T, then X^T -= Z^T (W X^T).  Rows are the queries of
// a tile (with softmax and values beside it), or, for the append, rows of the identity: then S is a row of every key of the tile
// carried to the chunk's END, and what is left of X at the chunk's start are the rows of H_{m-1} .. H_0.
// A wave has 16 rows; results stay in registers and are the next product's operand.  Bound by the fp32 matrix rate and, for few tiles, by the chain.
#include <type_traits>

#include "paged_decl.h"

namespace path {

constexpr int LDT = 68;      // row length of a 64 x 64 matrix in LDS
template <int D> constexpr size_t chunk_smem() { return (size_t)(3 * 64 * (D + 4) + 3 * 64 * LDT + 64 + 256) * 4; }

template <int D>
__global__ __launch_bounds__(512, 1) void paged_chunk_kernel(PagedArgs a) {
    constexpr int LD = D + 4;
    extern __shared__ __attribute__((aligned(16))) float sm[];
    float* const W = sm;
    float* const K = W + 64 * LD;
    float* const Q = K + 64 * LD;
    float* const B1 = Q + 64 * LD;
    float* const B2 = B1 + 64 * LDT;
    float* const B3 = B2 + 64 * LDT;
    float* const beta = B3 + 64 * LDT;
    float* const red = beta + 64;

    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, l32 = lane & 31, hh = lane >> 5;
    const int tile = blockIdx.x % a.tiles, h = blockIdx.x / a.tiles, Hq = a.H * a.G;
    int s = 0;
    for (int i = 0; i < a.nseq; i += 64) s += __popcll(__ballot(i + lane < a.nseq && first_tile(a, min(i + lane, a.nseq - 1)) <= tile));
    s = __builtin_amdgcn_readfirstlane(max(0, s - 1));
    const PagedSeq q = paged_seq(a, s);
    const int c = tile - first_tile(a, s), m = q.m - 64 * c;      // tokens from the tile's first on
    if (q.m <= a.few_limit || c < 0 || m <= 0) return;
    const int tok0 = q.t0 + 64 * c;

    const float* const kg = reinterpret_cast<const float*>(a.k);
    const float* const vg = reinterpret_cast<const float*>(a.v);
    const float* const wg = reinterpret_cast<const float*>(a.w);
    const float* const qg = reinterpret_cast<const float*>(a.q);
    auto stage = [&](float* dst, const float* src, int heads, int head) {
        for (int i = tid; i < 64 * D / 4; i += 512) {
            const int t = i / (D / 4), e = (i % (D / 4)) * 4;
            float x[4] = {0.f, 0.f, 0.f, 0.f};
            if (t < m) load_f32<4>(src + ((long long)(tok0 + t) * heads + head) * D + e, x);
            *reinterpret_cast<f32x4*>(dst + t * LD + e) = f32x4{x[0], x[1], x[2], x[3]};
        }
    };
    stage(W, wg, a.H, h);
    stage(K, kg, a.H, h);
    if (tid < 64) beta[tid] = tid < m ? reinterpret_cast<const float*>(a.beta)[(long long)(tok0 + tid) * a.H + h] : 0.f;
    if (a.cpages) {      // gate sums: c of the last cached token, the earlier tiles' gates, then one by one
        const float* const fg = reinterpret_cast<const float*>(a.log_f);
        if (tid < 256) {
            float x = 0.f;
            for (int t = tid; t < 64 * c; t += 256) x += fg[(long long)(q.t0 + t) * a.H + h];
            red[tid] = x;
        }
        __syncthreads();
        if (wv == 0) {
            float y = red[lane] + red[64 + lane] + red[128 + lane] + red[192 + lane];
            for (int o = 32; o; o >>= 1) y += __shfl_xor(y, o);
            const long long r = q.n > 0 ? paged_row(a, s, h, q.n - 1) : -1;
            y += r >= 0 ? a.cpages[r] : 0.f;
            float z = lane < m ? fg[(long long)(tok0 + lane) * a.H + h] : 0.f;
            for (int o = 1; o < 64; o <<= 1) { const float b = __shfl_up(z, o); if (lane >= o) z += b; }
            if (lane < m) a.crow[(long long)(tok0 + lane) * a.H + h] = y + z;
            if (a.append && lane < m) {
                const long long w = paged_row(a, s, h, q.n + 64 * c + lane);
                if (w >= 0) a.cpages[w] = y + z;
            }
        }
    }
    const size_t th = (size_t)tile * a.H + h;
    float* const kt = reinterpret_cast<float*>(a.kt) + th * 64 * D;
    float* const wt = reinterpret_cast<float*>(a.wt) + th * 64 * D;
    float* const zt = reinterpret_cast<float*>(a.zt) + th * 64 * D;
    float* const vt = reinterpret_cast<float*>(a.vt) + th * 64 * D;
    __syncthreads();

    for (int i = tid; i < 64 * D; i += 512) wt[(i / D) * D + (i % D)] = W[(i / D) * LD + i % D];
    if (a.attn)
        for (int i = tid; i < 64 * D; i += 512) {
            const int t = i / D, e = i % D;
            vt[e * 64 + (t)] = t < m ? vg[((long long)(tok0 + t) * a.H + h) * D + e] : 0.f;
        }
    if (a.append)
        for (int i = tid; i < 64 * (D / 4); i += 512) {
            const int t = i / (D / 4), e = (i % (D / 4)) * 4;
            const long long r = t < m ? paged_row(a, s, h, q.n + 64 * c + t) : -1;
            if (r >= 0) *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.vpages) + r * D + e) = *reinterpret_cast<const f32x4*>(vg + ((long long)(tok0 + t) * a.H + h) * D + e);
        }

    const bool low = wv < 4;                              // which of two 64 x 64 matrices
    const int rb = (wv >> 1) & 1, cb = wv & 1;            // this wave's 32 x 32 block of it
    auto put64 = [&](float* dst, const f32x16& v, auto f) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int r = 32 * rb + acc_row(j, hh), cc = 32 * cb + l32;
            dst[r * LDT + cc] = f(r, cc, v[j]);
        }
    };
    {   // N = diag(beta) strictLower(W W^T); D = strictLower(W K^T)
        f32x16 v = zero16();
        mm<float, D, false, false>(v, W, LD, 32 * rb, low ? W : K, LD, 32 * cb, l32, hh);
        if (low) {
            put64(B1, v, [&](int r, int cc, float x) { return cc < r ? beta[r] * x : 0.f; });
            put64(B2, v, [&](int, int, float) { return 0.f; });
        } else {
            put64(B3, v, [&](int r, int cc, float x) { return cc < r ? x : 0.f; });
        }
    }
    __syncthreads();
    // (I + N)^{-1} by blocks: 16 x 16 on the diagonal by substitution, a column per thread; then twice the lower left quarter, -T22 (N21 T11), by 16 x 16
    // blocks, a product's result the next one's right operand as it stands
    if (tid < 64) {
        const int b = tid & ~15, j = tid & 15;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float y = i == j ? 1.f : 0.f;
#pragma unroll
            for (int t = 0; t < i; ++t) y -= B1[(b + i) * LDT + b + t] * x[t];
            x[i] = y;
            B2[(b + i) * LDT + b + j] = y;
        }
    }
    __syncthreads();
    const int g = lane >> 4, c16 = lane & 15;
    auto quarter = [&](auto half, int b, int rq, int cq) {
        constexpr int HB = decltype(half)::value, NB = HB / 16;
        f32x4 tmp[NB];
#pragma unroll
        for (int r = 0; r < NB; ++r) {
            tmp[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < HB; k += 4)
                tmp[r] = __builtin_amdgcn_mfma_f32_16x16x4f32(B1[(b + HB + 16 * r + c16) * LDT + b + k + g], B2[(b + k + g) * LDT + b + 16 * cq + c16], tmp[r], 0, 0, 0);
        }
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < NB; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                y = __builtin_amdgcn_mfma_f32_16x16x4f32(B2[(b + HB + 16 * rq + c16) * LDT + b + HB + 16 * r + 4 * g + i], tmp[r][i], y, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) B2[(b + HB + 16 * rq + 4 * g + i) * LDT + b + 16 * cq + c16] = -y[i];
    };
    if (wv < 2) quarter(std::integral_constant<int, 16>(), 32 * wv, 0, 0);
    __syncthreads();
    if (wv < 4) quarter(std::integral_constant<int, 32>(), 0, wv >> 1, wv & 1);
    __syncthreads();
    for (int i = tid; i < 64 * 64; i += 512) B2[(i >> 6) * LDT + (i & 63)] *= beta[i & 63];      // T
    __syncthreads();
    if (low) {   // T D
        f32x16 v = zero16();
        mm<float, 64, false, true>(v, B2, LDT, 32 * rb, B3, LDT, 32 * cb, l32, hh);
        put64(B1, v, [&](int, int, float x) { return x; });
    } else {
        // -Z^T: rows of d, so computed with T W's factors exchanged
        for (int b = wv - 4; b < D / 32 * 2; b += 4) {
            const int r0 = 32 * (b >> 1), c0 = 32 * (b & 1);
            f32x16 v = zero16();
            mm<float, 64, true, false>(v, W, LD, r0, B2, LDT, c0, l32, hh);
#pragma unroll
            for (int j = 0; j < 16; ++j) zt[(r0 + acc_row(j, hh)) * 64 + c0 + l32] = -v[j];
        }
    }
    __syncthreads();
    for (int b = wv; b < D / 32 * 2; b += 8) {      // kt = K - (T D)^T W
        const int r0 = 32 * (b & 1), c0 = 32 * (b >> 1);
        f32x16 v = zero16();
        mm<float, 64, true, true>(v, B1, LDT, r0, W, LD, c0, l32, hh);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int r = r0 + acc_row(j, hh);
            kt[r * D + c0 + l32] = K[r * LD + c0 + l32] - v[j];
        }
    }
    if (!a.attn) return;
    for (int gq = 0; gq < a.G; ++gq) {
        const int hq = h * a.G + gq;
        __syncthreads();
        stage(Q, qg, Hq, hq);
        __syncthreads();
        if (low) {   // L = lower(Q W^T)
            f32x16 v = zero16();
            mm<float, D, false, false>(v, Q, LD, 32 * rb, W, LD, 32 * cb, l32, hh);
            put64(B3, v, [&](int r, int cc, float x) { return cc <= r ? x : 0.f; });
        }
        __syncthreads();
        f32x16 lt = zero16();
        if (low) {
            f32x16 v = zero16(), u = zero16();
            mm<float, D, false, false>(v, Q, LD, 32 * rb, K, LD, 32 * cb, l32, hh);
            mm<float, 64, false, true>(u, B3, LDT, 32 * rb, B1, LDT, 32 * cb, l32, hh);
            float* const sd = a.sd + ((size_t)tile * Hq + hq) * 4096;
#pragma unroll
            for (int j = 0; j < 16; ++j) sd[(32 * rb + acc_row(j, hh)) * 64 + 32 * cb + l32] = v[j] - u[j];
        } else {
            mm<float, 64, false, true>(lt, B3, LDT, 32 * rb, B2, LDT, 32 * cb, l32, hh);
        }
        __syncthreads();
        if (!low) put64(B3, lt, [&](int, int, float x) { return x; });
        __syncthreads();
        for (int b = wv; b < D / 32 * 2; b += 8) {      // X = Q - (L T) W
            const int r0 = 32 * (b & 1), c0 = 32 * (b >> 1);
            f32x16 v = zero16();
            mm<float, 64, false, true>(v, B3, LDT, r0, W, LD, c0, l32, hh);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int r = r0 + acc_row(j, hh);
                if (r < m) a.x[((long long)(tok0 + r) * Hq + hq) * D + c0 + l32] = Q[r * LD + c0 + l32] - v[j];
            }
        }
    }
}

// Products with 16 rows of results per wave whose right operand is packed from results.
template <int KD> struct SweepOperand {
    f32x4 f[KD / 16];
    __device__ __forceinline__ void pack(const f32x4* x) {
#pragma unroll
        for (int s = 0; s < KD / 16; ++s) f[s] = x[s];
    }
    __device__ __forceinline__ f32x4 left(const float* row, int g, f32x4 c) const {
#pragma unroll
        for (int s = 0; s < KD / 16; ++s) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(row + 16 * s + 4 * g);
#pragma unroll
            for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j], f[s][j], c, 0, 0, 0);
        }
        return c;
    }
};

template <int D, bool SCAN>
__global__ __launch_bounds__(256, 2) void paged_sweep_kernel(PagedArgs a) {
    constexpr int DT = D / 16;
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15, Hq = a.H * a.G;
    int s, h, hq = 0, tile, r0 = 0;
    if constexpr (SCAN) {
        int x = blockIdx.x;
        r0 = 64 * (x % (D / 64)); x /= D / 64;
        h = x % a.H;
        s = x / a.H;
        tile = 0;
    } else {
        tile = a.tiles - 1 - blockIdx.x / Hq;      // (the last tiles have the longest way)
        hq = blockIdx.x % Hq;
        h = hq / a.G;
        s = 0;
        for (int i = 0; i < a.nseq; i += 64) s += __popcll(__ballot(i + lane < a.nseq && first_tile(a, min(i + lane, a.nseq - 1)) <= tile));
        s = __builtin_amdgcn_readfirstlane(max(0, s - 1));
    }
    const PagedSeq q = paged_seq(a, s);
    if (q.m <= a.few_limit) return;
    const int first = first_tile(a, s), tiles = (q.m + 63) >> 6, ct = SCAN ? tiles : tile - first;
    if (ct < 0 || (!SCAN && ct >= tiles)) return;
    const int row = r0 + 16 * wv + c;                         // of the tile's queries, or of the identity
    const int tok = SCAN ? 0 : q.t0 + 64 * ct + row;
    const bool there = SCAN || 64 * ct + row < q.m;
    const long long at = (long long)tok * Hq + hq;

    f32x4 x[DT], O[SCAN ? 1 : DT];
    float m_run = -INFINITY, l_run = 0.f, cq = 0.f;
    const float sl2 = a.scale * LOG2E;
#pragma unroll
    for (int t = 0; t < DT; ++t) {
        x[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (SCAN) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[t][i] = 16 * t + 4 * g + i == row ? 1.f : 0.f;
        } else {
            if (there) x[t] = *reinterpret_cast<const f32x4*>(a.x + at * D + 16 * t + 4 * g);
            O[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    if (!SCAN && a.cpages && there) cq = a.crow[(long long)tok * a.H + h];

    auto attend = [&](int j, f32x4* S, bool own) {      // logits of tile j's keys: softmax and values
        float top = -INFINITY;
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = 16 * b + 4 * g + i;
                float y = S[b][i] * sl2;
                if (a.cpages) y += (cq - a.crow[(long long)min(q.t0 + 64 * j + key, a.T - 1) * a.H + h]) * LOG2E;
                if (own) y = key <= row ? y : -INFINITY;
                S[b][i] = y;
                top = fmaxf(top, y);
            }
        const float now = fmaxf(m_run, max_rows(top)), base = now == -INFINITY ? 0.f : now, f = __builtin_amdgcn_exp2f(m_run - base);
        m_run = now;
        float sum = 0.f;
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) { S[b][i] = __builtin_amdgcn_exp2f(S[b][i] - base); sum += S[b][i]; }
        l_run = l_run * f + sum;
        SweepOperand<64> P;
        P.pack(S);
        const float* const vt = reinterpret_cast<const float*>(a.vt) + ((size_t)(first + j) * a.H + h) * 64 * D;
#pragma unroll
        for (int t = 0; t < DT; ++t) O[t] = P.left(vt + (16 * t + c) * 64, g, O[t] * f);
    };
    if constexpr (!SCAN) {
        f32x4 S[4];
        const float* const sd = a.sd + ((size_t)tile * Hq + hq) * 4096 + row * 64;
#pragma unroll
        for (int b = 0; b < 4; ++b) S[b] = *reinterpret_cast<const f32x4*>(sd + 16 * b + 4 * g);
        attend(ct, S, true);
        if (__any(not_finite<DT>(O))) {      // a later token's infinity or NaN shows in the product with its weight 0: the values up to each row's own token again
#pragma unroll
            for (int t = 0; t < DT; ++t) O[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 16; ++k)
                for (int from = 0; from < 4; ++from) {
                    const int key = 16 * (k >> 2) + 4 * from + (k & 3);
                    const float p = __shfl(S[k >> 2][k & 3], 16 * from + c);
                    if (!there || key > row) continue;
                    const float* const v = reinterpret_cast<const float*>(a.v) + ((long long)(q.t0 + 64 * ct + key) * a.H + h) * D + 4 * g;
#pragma unroll
                    for (int t = 0; t < DT; ++t) {
                        const f32x4 x = *reinterpret_cast<const f32x4*>(v + 16 * t);
#pragma unroll
                        for (int i = 0; i < 4; ++i) O[t][i] += p * x[i];
                    }
                }
        }
    }
    for (int j = ct - 1; j >= 0; --j) {
        const size_t th = ((size_t)(first + j) * a.H + h) * 64 * D;
        const float* const kt = reinterpret_cast<const float*>(a.kt) + th;
        const float* const wt = reinterpret_cast<const float*>(a.wt) + th;
        const float* const zt = reinterpret_cast<const float*>(a.zt) + th;
        SweepOperand<D> X;
        X.pack(x);
        f32x4 S[4], Y[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            S[b] = X.left(kt + (16 * b + c) * D, g, f32x4{0.f, 0.f, 0.f, 0.f});
            Y[b] = X.left(wt + (16 * b + c) * D, g, f32x4{0.f, 0.f, 0.f, 0.f});
        }
        SweepOperand<64> YB;
        YB.pack(Y);
#pragma unroll
        for (int t = 0; t < DT; ++t) x[t] = YB.left(zt + (16 * t + c) * 64, g, x[t]);
        if constexpr (SCAN) {
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = 64 * j + 16 * b + 4 * g + i;
                    const long long r = t < q.m ? paged_row(a, s, h, q.n + t) : -1;
                    if (r >= 0) reinterpret_cast<float*>(a.kpages)[r * D + row] = S[b][i];
                }
        } else {
            attend(j, S, false);
        }
    }
    if constexpr (SCAN) {
        float* const p = reinterpret_cast<float*>(a.pt) + (((size_t)s * a.H + h) * D + row) * D;
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            f32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = (x[t][i] - (16 * t + 4 * g + i == row ? 1.f : 0.f));
            *reinterpret_cast<f32x4*>(p + 16 * t + 4 * g) = v;
        }
    } else {
        l_run = sum_rows(l_run);
        if (there && q.n == 0) {      // nothing cached: that was all
            const float inv = 1.f / l_run;
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                f32x4 v;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = (O[t][i] * inv);
                *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.o) + at * D + 16 * t + 4 * g) = v;
            }
            if (g == 0) a.lse[at] = (m_run + __builtin_amdgcn_logf(l_run)) * LN2;
        } else if (there) {
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                *reinterpret_cast<f32x4*>(a.x + at * D + 16 * t + 4 * g) = x[t];
                *reinterpret_cast<f32x4*>(a.many_o + at * D + 16 * t + 4 * g) = O[t];
            }
            if (g == 0) { a.many_ml[2 * at] = m_run; a.many_ml[2 * at + 1] = l_run; }
        }
    }
}

template <int D>
static hipError_t launch_chunk_t(const PagedArgs& a, hipStream_t st) {
    constexpr size_t bytes = chunk_smem<D>();
    static_assert(bytes <= 160 * 1024, "LDS");
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_chunk_kernel<D>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL((paged_chunk_kernel<D>), dim3((unsigned)(a.tiles * a.H)), dim3(512), bytes, st, a);
    return hipGetLastError();
}
hipError_t launch_paged_chunk(const PagedArgs& a, int d, hipStream_t st) { return d == 64 ? launch_chunk_t<64>(a, st) : launch_chunk_t<128>(a, st); }
template <int D, bool SCAN>
static hipError_t launch_sweep_t(const PagedArgs& a, hipStream_t st) {
    const unsigned grid = SCAN ? (unsigned)(a.nseq * a.H * (D / 64)) : (unsigned)(a.tiles * a.H * a.G);
    hipLaunchKernelGGL((paged_sweep_kernel<D, SCAN>), dim3(grid), dim3(256), 0, st, a);
    return hipGetLastError();
}
hipError_t launch_paged_sweep(const PagedArgs& a, int d, hipStream_t st) { return d == 64 ? launch_sweep_t<64, false>(a, st) : launch_sweep_t<128, false>(a, st); }
hipError_t launch_paged_scan(const PagedArgs& a, int d, hipStream_t st) { return d == 64 ? launch_sweep_t<64, true>(a, st) : launch_sweep_t<128, true>(a, st); }

}  // namespace path
