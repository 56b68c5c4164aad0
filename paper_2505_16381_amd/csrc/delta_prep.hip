// Gated delta rule: the matrices of a chunk, all chunks at once (delta_decl.h has the formulas).
#include <type_traits>

#include "delta_parts.h"

namespace path {

static constexpr int DP_LF = 68;      // floats in a row of a 64 x 64 matrix in LDS

// c += A B, 16x16 blocks (bi, bk) and (bk, bj) of fp32 matrices in LDS
__device__ __forceinline__ f32x4 block_mma(const float* A, int bi, int bk, const float* B, int bj, int n, int g, f32x4 c) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(A + (16 * bi + n) * DP_LF + 16 * bk + 4 * g);
    f32x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = B[(16 * bk + 4 * g + e) * DP_LF + 16 * bj + n];
    return DeltaOps<float>::mma(x, y, c);
}
// the same with B in registers, as a product left it
__device__ __forceinline__ f32x4 block_mma(const float* A, int bi, int bk, f32x4 y, int n, int g, f32x4 c) {
    return DeltaOps<float>::mma(*reinterpret_cast<const f32x4*>(A + (16 * bi + n) * DP_LF + 16 * bk + 4 * g), y, c);
}

// K K^T and Q K^T take the caller's numbers as they are
__device__ __forceinline__ f32x4 mma_user(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma_user(f32x4 a, f32x4 b, f32x4 c) { return DeltaOps<float>::mma(a, b, c); }

template <typename T>
__device__ __forceinline__ void store_frags(const float* X, bool transposed, void* out, size_t unit, int tid) {
    typedef DeltaOps<T> P;
    constexpr int NP = P::NP;
    typename P::Frag* const dst = reinterpret_cast<typename P::Frag*>(out) + unit * NP * P::NLOW * 64;
    constexpr int NT = 64 / 16, NS = 64 / P::SL;
    for (int i = tid; i < P::NLOW * 64; i += 256) {
        const int fr = i >> 6, lane = i & 63, n = lane & 15, g = lane >> 4;
        int t = 0, s = 0;
#pragma unroll
        for (int tt = 0; tt < NT; ++tt)
#pragma unroll
            for (int ss = 0; ss < NS; ++ss)
                if (transposed ? P::up(tt, ss) && P::up_at(tt, ss) == fr : P::low(tt, ss) && P::low_at(tt, ss) == fr) { t = tt; s = ss; }
        const int r = P::row(t, n), k = P::SL * s + P::FE * g;
        float x[P::FE];
#pragma unroll
        for (int e = 0; e < P::FE; ++e) x[e] = transposed ? X[(k + e) * DP_LF + r] : X[r * DP_LF + k + e];
        DeltaParts<T, NP> o;
        delta_split<T, NP>(x, o);
#pragma unroll
        for (int p = 0; p < NP; ++p) dst[p * P::NLOW * 64 + i] = o.p[p];
    }
}

// 16 bytes of row r of a tokens' matrix, zeros behind the last one
template <typename F, typename T> __device__ __forceinline__ F row_frag(const T* p, long long ld, int r, int left, int x) {
    F f;
#pragma unroll
    for (int e = 0; e < 16 / (int)sizeof(T); ++e) f[e] = (T)0.f;
    return r < left ? *reinterpret_cast<const F*>(p + r * ld + x) : f;
}

// Four waves to a chunk, 16 rows each; K and Q come from memory as operands (a wave's four tiles of K overlap the others' in L1).  Bound by the chain of its phases,
// so by how many workgroups a CU holds: LDS has the 64 x 64 matrices alone, and 128 registers (three of them spilled, of fp32 at d = 128 eight) let four in.  d = 128, 8192 tokens of 64 heads: 119 us, 4.0 TB/s
// (K, Q in, P, M out: 478 MB; with operands of one part 108, where three workgroups took 120).  With the transposes for training 176 us (three workgroups: a third matrix in LDS).
template <typename T, int D, bool TRAIN>      // TRAIN: the transposes, for the gradients
__global__ __launch_bounds__(256, TRAIN ? 3 : 4) void delta_prep_kernel(DeltaArgs a) {
    typedef typename std::conditional<sizeof(T) == 2, half_t, float>::type C;      // of the operands that are kept
    typedef typename Tr<T>::Frag Frag;
    constexpr int SL = sizeof(T) == 2 ? 32 : 16, FE = 16 / (int)sizeof(T);
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    float* const N = reinterpret_cast<float*>(smem);
    float* const M = N + 64 * DP_LF;
    float* const rows = M + 64 * DP_LF;
    float* const Lm = rows + DELTA_ROWS * 64;      // training only
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const int tile = __builtin_amdgcn_readfirstlane(blockIdx.x / a.V), hv = blockIdx.x - tile * a.V, hk = __builtin_amdgcn_readfirstlane(hv / a.G);
    int s, c;
    DeltaSeq sq;
    if (!delta_tile(a, tile, lane, s, c, sq)) return;
    const int t0 = c * CHUNK, left = sq.len - t0;      // tokens of this chunk: min(64, left)
    const size_t unit = (size_t)tile * a.V + hv;
    const long long kat = delta_at(a, sq, s, a.ks, a.kt) + hk * a.kh + t0 * a.kt, sat = delta_at(a, sq, s, a.ss, a.st) + hv * a.sh + t0 * a.st;
    const T *const kp = static_cast<const T*>(a.k) + kat, *const qp = static_cast<const T*>(a.q) + kat;

    // rows 16 wv .. of K K^T and Q K^T
    Frag fk[D / SL], fq[D / SL];
#pragma unroll
    for (int x = 0; x < D / SL; ++x) fk[x] = row_frag<Frag>(kp, a.kt, 16 * wv + n, left, x * SL + FE * g);
#pragma unroll
    for (int x = 0; x < D / SL; ++x) fq[x] = row_frag<Frag>(qp, a.kt, 16 * wv + n, left, x * SL + FE * g);
    if (wv == 0) {
        // Running sums in 64 bits: 64 gates of -20 each add up to 1e3, whose rounding to 32 bits would be 6e-5 of a neighbour's weight.  Gates below exp(-200) count as
        // that: it is nothing beside any number of 32 bits, and sums stay small enough for differences between the tokens behind a gate that forgets everything.
        const bool in = lane < left;
        const float be = in ? (float)static_cast<const T*>(a.beta)[sat + lane * a.st] : 0.f;
        float lf = in && a.log_f ? (float)static_cast<const T*>(a.log_f)[sat + lane * a.st] : 0.f;
        lf = lf < -200.f ? -200.f : lf;
        double b = lf;
#pragma unroll
        for (int x = 1; x < 64; x *= 2) {
            const double y = __shfl_up(b, x);
            if (lane >= x) b += y;
        }
        const double last = __shfl(b, 63);
        const float hi = (float)b, vals[DELTA_ROWS] = {be, expf(hi), expf((float)(last - b)), hi, (float)(b - (double)hi)};
        float* const out = a.rows + unit * DELTA_ROWS * 64;
#pragma unroll
        for (int i = 0; i < DELTA_ROWS; ++i) { rows[i * 64 + lane] = vals[i]; out[i * 64 + lane] = vals[i]; }
    }
    f32x4 kk[4], qk[4];
#pragma unroll
    for (int ib = 0; ib < 4; ++ib) {
        kk[ib] = qk[ib] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (ib <= wv) {
            Frag f[D / SL];
#pragma unroll
            for (int z = 0; z < D / SL; ++z) f[z] = ib == wv ? fk[z] : row_frag<Frag>(kp, a.kt, 16 * ib + n, left, z * SL + FE * g);
#pragma unroll
            for (int z = 0; z < D / SL; ++z) {
                kk[ib] = mma_user(fk[z], f[z], kk[ib]);
                qk[ib] = mma_user(fq[z], f[z], qk[ib]);
            }
        }
    }
    __syncthreads();
    {
        float bh[4], bl[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) { const int r = 16 * wv + 4 * g + j; bh[j] = rows[3 * 64 + r]; bl[j] = rows[4 * 64 + r]; }
#pragma unroll
        for (int ib = 0; ib < 4; ++ib) {
            const int i = 16 * ib + n;
            const float ih = rows[3 * 64 + i], il = rows[4 * 64 + i], be = rows[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = 16 * wv + 4 * g + j;
                const float w = ib <= wv ? expf((bh[j] - ih) + (bl[j] - il)) : 0.f, l = i < r ? w * kk[ib][j] : 0.f;
                N[r * DP_LF + i] = l * be;
                M[r * DP_LF + i] = i <= r ? a.scale * w * qk[ib][j] : 0.f;
                if (TRAIN) Lm[r * DP_LF + i] = l;
            }
        }
    }
    __syncthreads();

    // P = (I + N)^-1: 16x16 diagonal blocks by substitution, a column per lane, then -X22 N21 X11, of 16 and of 32 rows, all in 32 bits
    {
        float x[16];
        const float* const B = N + 16 * wv * DP_LF + 16 * wv;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float y = r == n ? 1.f : 0.f;
#pragma unroll
            for (int i = 0; i < r; ++i) y -= B[r * DP_LF + i] * x[i];
            x[r] = y;
        }
        __builtin_amdgcn_wave_barrier();
        if (g == 0) {
#pragma unroll
            for (int r = 0; r < 16; ++r) N[(16 * wv + r) * DP_LF + 16 * wv + n] = x[r];
        }
    }
    __syncthreads();
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    if (wv < 2) {
        const f32x4 y = block_mma(N, 2 * wv + 1, 2 * wv, N, 2 * wv, n, g, zero), x = block_mma(N, 2 * wv + 1, 2 * wv + 1, y, n, g, zero);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < 4; ++j) N[(32 * wv + 16 + 4 * g + j) * DP_LF + 32 * wv + n] = -x[j];
    }
    __syncthreads();
    {
        const int bi = 2 + (wv >> 1), bj = wv & 1;
        f32x4 x = zero;
#pragma unroll
        for (int k = 2; k < 4; ++k) {
            if (k > bi) continue;
            f32x4 y = zero;
#pragma unroll
            for (int l = 0; l < 2; ++l)
                if (l >= bj) y = block_mma(N, k, l, N, bj, n, g, y);
            x = block_mma(N, bi, k, y, n, g, x);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) N[(16 * bi + 4 * g + j) * DP_LF + 16 * bj + n] = -x[j];
    }
    __syncthreads();
    store_frags<C>(N, false, a.p, unit, tid);
    store_frags<C>(M, false, a.m, unit, tid);
    if constexpr (TRAIN) {
        store_frags<C>(M, true, a.mt, unit, tid);
        // A = I - diag(beta) P L, rows 16 wv ..
        f32x4 x[4];
#pragma unroll
        for (int bj = 0; bj < 4; ++bj) {
            x[bj] = zero;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k >= bj && k <= wv) x[bj] = block_mma(N, wv, k, Lm, bj, n, g, x[bj]);
        }
        __syncthreads();
#pragma unroll
        for (int bj = 0; bj < 4; ++bj)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = 16 * wv + 4 * g + j, i = 16 * bj + n;
                N[r * DP_LF + i] = (r == i ? 1.f : 0.f) - rows[r] * x[bj][j];
            }
        __syncthreads();
        store_frags<C>(N, true, a.at, unit, tid);
    }
}

template <typename T, int D, bool TRAIN>
static hipError_t launch(const DeltaArgs& a, hipStream_t stream) {
    constexpr size_t bytes = (size_t)((TRAIN ? 3 : 2) * 64 * DP_LF + DELTA_ROWS * 64) * 4;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&delta_prep_kernel<T, D, TRAIN>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (attr != hipSuccess) return attr;
    delta_prep_kernel<T, D, TRAIN><<<dim3((unsigned)a.tiles * a.V), dim3(256), bytes, stream>>>(a);
    return hipGetLastError();
}
template <int D>
static hipError_t launch_d(const DeltaArgs& a, int is_bf16, bool training, hipStream_t stream) {
    if (!is_bf16) return training ? launch<float, D, true>(a, stream) : launch<float, D, false>(a, stream);
    return training ? launch<bf16_t, D, true>(a, stream) : launch<bf16_t, D, false>(a, stream);
}
hipError_t launch_delta_prep(const DeltaArgs& a, int d, int is_bf16, bool training, hipStream_t stream) {
    return d == 64 ? launch_d<64>(a, is_bf16, training, stream) : launch_d<128>(a, is_bf16, training, stream);
}

}  // namespace path
