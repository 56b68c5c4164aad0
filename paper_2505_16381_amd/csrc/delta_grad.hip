// Gated delta rule: gradients of q, k, beta and log f from the states, their gradients, U and Y of a chunk, all chunks at once (delta_decl.h has the formulas).
// A workgroup takes a chunk of a key head and adds up its value heads one after the other, in registers.
#include "delta_parts.h"

namespace path {

// ---- fp32: 16x16 products; K, Q, dO in LDS, the rest as fragments from memory ----

static constexpr int DG_LF = 68;

template <int D>
__global__ __launch_bounds__(256) void delta_grad_kernel(DeltaArgs a) {
    typedef DeltaOps<float> P;
    constexpr int LD = D + 4, NR = D / 16;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    float* const K = reinterpret_cast<float*>(smem);
    float *const Q = K + 64 * LD, *const O = Q + 64 * LD, *const Gq = O + 64 * LD, *const Gk = Gq + 64 * DG_LF, *const rows = Gk + 64 * DG_LF, *const red = rows + DELTA_ROWS * 64;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, n = lane & 15, g = lane >> 4;
    const int tile = __builtin_amdgcn_readfirstlane(blockIdx.x / a.H), hk = blockIdx.x - tile * a.H;
    int s, c;
    DeltaSeq sq;
    if (!delta_tile(a, tile, lane, s, c, sq)) return;
    const int t0 = c * CHUNK, left = sq.len - t0;
    const long long kat = delta_at(a, sq, s, a.ks, a.kt) + hk * a.kh + t0 * a.kt;
    const float *const kp = static_cast<const float*>(a.k) + kat, *const qp = static_cast<const float*>(a.q) + kat;
    auto fill = [&](float* to, const float* from, long long ld) {
        for (int i = tid; i < 64 * D / 4; i += 256) {
            const int r = i / (D / 4), x = i % (D / 4) * 4;
            *reinterpret_cast<f32x4*>(to + r * LD + x) = r < left ? *reinterpret_cast<const f32x4*>(from + r * ld + x) : f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    fill(K, kp, a.kt);
    fill(Q, qp, a.kt);
    f32x4 dq[NR], dk[NR];
#pragma unroll
    for (int t = 0; t < NR; ++t) dq[t] = dk[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    // fragments: rows along lanes, contraction along the row, or (tr) rows of the product along the matrix's columns
    auto nat = [&](const float* X, int ld, int r0, int k0) { return *reinterpret_cast<const f32x4*>(X + (size_t)(r0 + n) * ld + k0 + 4 * g); };
    auto tr = [&](const float* X, int ld, int r0, int k0) {
        f32x4 f;
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = X[(size_t)(k0 + 4 * g + e) * ld + r0 + n];
        return f;
    };
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const int r0 = 16 * wv;
#pragma unroll 1
    for (int x = 0; x < a.G; ++x) {
        const int hv = hk * a.G + x;
        const size_t u = (size_t)tile * a.V + hv;
        const long long vat = delta_at(a, sq, s, a.vs, a.vt) + hv * a.vh + t0 * a.vt, sat = delta_at(a, sq, s, a.ss, a.st) + hv * a.sh + t0 * a.st;
        const float *const S = static_cast<const float*>(a.sm) + u * D * D, *const G = static_cast<const float*>(a.gm) + u * D * D;
        const float *const U = static_cast<const float*>(a.um) + u * D * 64, *const Y = static_cast<const float*>(a.ym) + u * D * 64;
        __syncthreads();
        fill(O, static_cast<const float*>(a.d_o) + vat, a.vt);
        for (int i = tid; i < DELTA_ROWS * 64; i += 256) rows[i] = a.rows[u * DELTA_ROWS * 64 + i];
        float sg = 0.f;      // <S, G>
        for (int i = tid; i < D * D; i += 256) sg += S[i] * G[i];
        __syncthreads();
        float be[4], ga[4], rh[4], bh[4], bl[4], db[4], dl[4], kug = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = r0 + 4 * g + j;
            be[j] = rows[r]; ga[j] = rows[64 + r]; rh[j] = rows[128 + r]; bh[j] = rows[192 + r]; bl[j] = rows[256 + r];
            db[j] = dl[j] = 0.f;
        }
#pragma unroll
        for (int ib = 0; ib < 4; ++ib) {
            f32x4 X = zero, N = zero, KK = zero;
            if (ib <= wv)
#pragma unroll 1
                for (int z = 0; z < D; z += 16) {
                    const f32x4 uf = tr(U, 64, 16 * ib, z);
                    X = P::mma(tr(Y, 64, r0, z), uf, X);
                    N = P::mma(nat(O, LD, r0, z), uf, N);
                    KK = P::mma(nat(K, LD, r0, z), nat(K, LD, 16 * ib, z), KK);
                }
            const int i = 16 * ib + n;
            const float ih = rows[192 + i], il = rows[256 + i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = r0 + 4 * g + j;
                const float w = expf((bh[j] - ih) + (bl[j] - il));
                Gq[r * DG_LF + i] = i <= r ? a.scale * w * N[j] : 0.f;
                Gk[r * DG_LF + i] = i < r ? -be[j] * w * X[j] : 0.f;
                if (i < r) db[j] -= X[j] * w * KK[j];
            }
        }
        // Y.v, value indices n, n + 16, ..
        const float* const vp = static_cast<const float*>(a.v) + vat;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = r0 + 4 * g + j;
            if (r < left)
                for (int z = n; z < D; z += 16) db[j] += Y[z * 64 + r] * vp[r * a.vt + z];
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < NR; ++t) {
            f32x4 ys = zero, os = zero, ug = zero, q1 = zero, rd = zero, wr = zero;
#pragma unroll 1
            for (int z = 0; z < D; z += 16) {
                const f32x4 sf = tr(S, D, 16 * t, z);
                ys = P::mma(tr(Y, 64, r0, z), sf, ys);
                os = P::mma(nat(O, LD, r0, z), sf, os);
                ug = P::mma(tr(U, 64, r0, z), tr(G, D, 16 * t, z), ug);
            }
#pragma unroll 1
            for (int z = 0; z < 64; z += 16) {
                const f32x4 kf = tr(K, LD, 16 * t, z);
                q1 = P::mma(nat(Gq, DG_LF, r0, z), kf, q1);
                rd = P::mma(nat(Gk, DG_LF, r0, z), kf, rd);
                wr = P::mma(tr(Gk, DG_LF, r0, z), kf, wr);
                wr = P::mma(tr(Gq, DG_LF, r0, z), tr(Q, LD, 16 * t, z), wr);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = r0 + 4 * g + j;
                const float kv = K[r * LD + 16 * t + n], qv = Q[r * LD + 16 * t + n];
                const float dqv = q1[j] + a.scale * ga[j] * os[j], rdv = rd[j] - ga[j] * be[j] * ys[j], u4 = rh[j] * ug[j], wrv = wr[j] + u4;
                db[j] -= ga[j] * ys[j] * kv;
                dl[j] += qv * dqv + kv * (rdv - wrv);
                kug += kv * u4;
                dq[t][j] += dqv;
                dk[t][j] += rdv + wrv;
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int z = 1; z < 16; z *= 2) { db[j] += __shfl_xor(db[j], z); dl[j] += __shfl_xor(dl[j], z); }
        kug += rows[64 + 63] * sg;
#pragma unroll
        for (int z = 1; z < 64; z *= 2) kug += __shfl_xor(kug, z);
        if (lane == 0) red[wv] = kug;
        if (n == 0)
#pragma unroll
            for (int j = 0; j < 4; ++j) { red[64 + r0 + 4 * g + j] = db[j]; red[128 + r0 + 4 * g + j] = dl[j]; }
        __syncthreads();
        if (wv == 0) {
            float l = red[128 + lane];
#pragma unroll
            for (int z = 1; z < 64; z *= 2) {
                const float y = __shfl_down(l, z);
                if (lane + z < 64) l += y;
            }
            if (lane < left) {
                static_cast<float*>(a.dbeta)[sat + lane * a.st] = red[64 + lane];
                if (a.dlog_f) static_cast<float*>(a.dlog_f)[sat + lane * a.st] = l + ((red[0] + red[1]) + (red[2] + red[3]));
            }
        }
    }
    float *const dqp = static_cast<float*>(a.dq) + kat, *const dkp = static_cast<float*>(a.dk) + kat;
#pragma unroll
    for (int t = 0; t < NR; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = r0 + 4 * g + j;
            if (r < left) {
                dqp[r * a.kt + 16 * t + n] = dq[t][j];
                dkp[r * a.kt + 16 * t + n] = dk[t][j];
            }
        }
}

// ---- bf16: 32x32 products of fp16 operands, each matrix over a power of two of its own ----
//
// Operands of one part: the states, U, Y and dO with the exponents of their largest values taken out (numbers down to 2^-24 of those keep eleven bits), so that gradients of any
// size are as exact: results come out 2e-4 (of their norm) off before they are rounded to bf16, 2e-3.  bf16 operands of one part: dk 2.5e-3, dlog_f 2.2e-3 off.

// sums over the 32 lanes of a half-wave of each of 16 values; lane l32 gets the value l32 / 2
__device__ __forceinline__ float sum16(float (&v)[16], int l32) {
#pragma unroll
    for (int w = 8, m = 16; w >= 1; w /= 2, m /= 2) {
        const bool up = l32 & m;
#pragma unroll
        for (int j = 0; j < w; ++j) {
            const float keep = up ? v[j + w] : v[j], give = up ? v[j] : v[j + w];
            v[j] = keep + __shfl_xor(give, m);
        }
    }
    return v[0] + __shfl_xor(v[0], 1);
}
__device__ __forceinline__ half_t half_power(int e) { return e < -24 ? (half_t)0.f : (half_t)ldexpf(1.f, e); }

template <int D> struct Grad16 {
    static constexpr int NT = 4 * D, NWV = NT / 64, LD = D + 8, LU = 72, CB = D / 32;
    static constexpr int K = 0, Q = K + 64 * LD, O = Q + 64 * LD, U = O + 64 * LD, Y = U + D * LU, S = Y + D * LU, GQ = S + D * LD, GK = GQ + 64 * LU, HALVES = GK + 64 * LU;
    static constexpr size_t bytes = (size_t)HALVES * 2 + (DELTA_ROWS * 64 + 32 + 64 * (2 * CB + 2 + NWV)) * 4;
};

template <int D>
__global__ __launch_bounds__(Grad16<D>::NT, 1) void delta_grad16_kernel(DeltaArgs a) {
    typedef Grad16<D> C;
    constexpr int NT = C::NT, LD = C::LD, LU = C::LU, CB = C::CB, NWV = C::NWV;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    half_t* const H = reinterpret_cast<half_t*>(smem);
    half_t *const K = H + C::K, *const Q = H + C::Q, *const O = H + C::O, *const U = H + C::U, *const Y = H + C::Y, *const S = H + C::S, *const Gq = H + C::GQ, *const Gk = H + C::GK;
    float* const rows = reinterpret_cast<float*>(H + C::HALVES);
    float *const wred = rows + DELTA_ROWS * 64;      // [2][16] of the waves
    float *const kys = wred + 32, *const dls = kys + 64 * CB, *const xl = dls + 64 * CB, *const yv = xl + 128;      // [column block][64], the same, [2][64], [wave][64]
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tile = __builtin_amdgcn_readfirstlane(blockIdx.x / a.H), hk = blockIdx.x - tile * a.H;
    int s, c;
    DeltaSeq sq;
    if (!delta_tile(a, tile, lane, s, c, sq)) return;
    const int t0 = c * CHUNK, left = sq.len - t0;
    const long long kat = delta_at(a, sq, s, a.ks, a.kt) + hk * a.kh + t0 * a.kt;
    constexpr int PPR = D / 8, NP = 64 * PPR / NT, NU = D * 8 / NT, NS = D * PPR / NT;      // pieces of 8 in a row; of a thread: tokens' matrices, U and Y, states
    auto rows_in = [&](const void* base, long long ld, int i) {      // piece i of the thread of a tokens' matrix
        const int p = tid + i * NT, r = p / PPR, x = p % PPR * 8;
        bf16x8 f;
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (bf16_t)0.f;
        if (r < left) f = *reinterpret_cast<const bf16x8*>(static_cast<const bf16_t*>(base) + r * ld + x);
        return f;
    };
    auto put = [&](half_t* to, const bf16x8& f, int i, float w) {
        const int p = tid + i * NT, r = p / PPR, x = p % PPR * 8;
        halfx8 y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (half_t)((float)f[e] * w);
        *reinterpret_cast<halfx8*>(to + r * LD + x) = y;
    };
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        put(K, rows_in(static_cast<const bf16_t*>(a.k) + kat, a.kt, i), i, 1.f);
        put(Q, rows_in(static_cast<const bf16_t*>(a.q) + kat, a.kt, i), i, 1.f);
    }
    const int rb = wv / CB, cb = wv % CB;      // the wave's 32 tokens and 32 key indices of dq, dk
    f32x16 dq = zero16(), dk = zero16();
#pragma unroll 1
    for (int x = 0; x < a.G; ++x) {
        const int hv = hk * a.G + x;
        // (the lane's place, made anew: LDS addresses of all products kept across the loop over heads would not fit the registers)
        int l32 = lane & 31, h = lane >> 5;
        asm volatile("" : "+v"(l32), "+v"(h));
        const size_t u = (size_t)tile * a.V + hv;
        const long long vat = delta_at(a, sq, s, a.vs, a.vt) + hv * a.vh + t0 * a.vt, sat = delta_at(a, sq, s, a.ss, a.st) + hv * a.sh + t0 * a.st;
        const half_t *const sg = static_cast<const half_t*>(a.sm) + u * D * D, *const gg = static_cast<const half_t*>(a.gm) + u * D * D;
        const half_t *const ug = static_cast<const half_t*>(a.um) + u * D * 64, *const yg = static_cast<const half_t*>(a.ym) + u * D * 64;
        bf16x8 of[NP];
        halfx8 sf[NS], gf[NS], uf[NU], yf[NU];
#pragma unroll
        for (int i = 0; i < NP; ++i) of[i] = rows_in(static_cast<const bf16_t*>(a.d_o) + vat, a.vt, i);
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            uf[i] = *reinterpret_cast<const halfx8*>(ug + (tid + i * NT) * 8);
            yf[i] = *reinterpret_cast<const halfx8*>(yg + (tid + i * NT) * 8);
        }
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            sf[i] = *reinterpret_cast<const halfx8*>(sg + (tid + i * NT) * 8);
            gf[i] = *reinterpret_cast<const halfx8*>(gg + (tid + i * NT) * 8);
        }
        const int *const vex = a.vex + ((size_t)s * a.V + hv) * 8, *const gex = a.gex + ((size_t)s * a.V + hv) * 8;
        int ev = vex[0], eg = gex[0];      // the largest exponents: of S and U, of G, Y and dO
#pragma unroll
        for (int b = 1; b < D / 16; ++b) {
            ev = vex[b] > ev ? vex[b] : ev;
            eg = gex[b] > eg ? gex[b] : eg;
        }
        __syncthreads();      // (the head before has been read out)
        for (int i = tid; i < DELTA_ROWS * 64; i += NT) rows[i] = a.rows[u * DELTA_ROWS * 64 + i];
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int p = tid + i * NT, r = p >> 3, y = (p & 7) * 8;
            const half_t wu = half_power(vex[r >> 4] - ev), wy = half_power(gex[r >> 4] - eg);
            *reinterpret_cast<halfx8*>(U + r * LU + y) = uf[i] * wu;
            *reinterpret_cast<halfx8*>(Y + r * LU + y) = yf[i] * wy;
        }
        float sum = 0.f;      // <S, G>, over 2^(ev + eg)
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            const int p = tid + i * NT, r = p / PPR, y = p % PPR * 8;
            sf[i] = sf[i] * half_power(vex[r >> 4] - ev);
            gf[i] = gf[i] * half_power(gex[r >> 4] - eg);
            *reinterpret_cast<halfx8*>(S + r * LD + y) = sf[i];
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += (float)sf[i][e] * (float)gf[i][e];
        }
        const float wo = delta_power(-eg);
#pragma unroll
        for (int i = 0; i < NP; ++i) put(O, of[i], i, wo);
        __syncthreads();

        // X, N, K K^T of the lower 32x32 blocks -> Gk, Gq, sum_i X_ri L_ri
#pragma unroll 1
        for (int job = wv; job < 6; job += NWV) {
            const int b = job % 3, br = b ? 1 : 0, bi = b == 2 ? 1 : 0;
            f32x16 acc = zero16();
            if (job < 3) {
                mm<half_t, D, true, true>(acc, Y, LU, 32 * br, U, LU, 32 * bi, l32, h);
                __builtin_amdgcn_sched_barrier(0);
                f32x16 kk = zero16();
                mm<half_t, D, false, false>(kk, K, LD, 32 * br, K, LD, 32 * bi, l32, h);
                float part[16];
                const int i = 32 * bi + l32;
                const float ih = rows[192 + i], il = rows[256 + i];
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int r = 32 * br + acc_row(j, h);
                    const float w = expf((rows[192 + r] - ih) + (rows[256 + r] - il));
                    const bool in = i < r;
                    part[j] = in ? acc[j] * w * kk[j] : 0.f;
                    Gk[r * LU + i] = (half_t)(in ? -rows[r] * w * acc[j] * 0x1p-12f : 0.f);
                }
                if (b == 1)
#pragma unroll
                    for (int j = 0; j < 16; ++j) Gk[acc_row(j, h) * LU + 32 + l32] = (half_t)0.f;
                const float y = sum16(part, l32);
                if (!(l32 & 1)) xl[bi * 64 + 32 * br + acc_row(l32 >> 1, h)] = y;
                if (b == 0 && lane < 32) xl[64 + lane] = 0.f;
            } else {
                mm<half_t, D, false, true>(acc, O, LD, 32 * br, U, LU, 32 * bi, l32, h);
                const int i = 32 * bi + l32;
                const float ih = rows[192 + i], il = rows[256 + i];
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int r = 32 * br + acc_row(j, h);
                    const float w = expf((rows[192 + r] - ih) + (rows[256 + r] - il));
                    Gq[r * LU + i] = (half_t)(i <= r ? w * acc[j] * 0x1p-12f : 0.f);
                }
                if (b == 1)
#pragma unroll
                    for (int j = 0; j < 16; ++j) Gq[acc_row(j, h) * LU + 32 + l32] = (half_t)0.f;
            }
        }
        {      // Y.v of token `lane`, the wave's share of the value indices
            float y = 0.f;
            if (lane < left) {
                constexpr int W = D / NWV;
                const bf16_t* const vp = static_cast<const bf16_t*>(a.v) + vat + lane * a.vt + wv * W;
#pragma unroll
                for (int z = 0; z < W; z += 8) {
                    const bf16x8 f = *reinterpret_cast<const bf16x8*>(vp + z);
#pragma unroll
                    for (int e = 0; e < 8; ++e) y += (float)f[e] * (float)Y[(wv * W + z + e) * LU + lane];
                }
            }
            yv[wv * 64 + lane] = y;
        }
        f32x16 ys = zero16(), os = zero16();
        __builtin_amdgcn_sched_barrier(0);
        mm<half_t, D, true, true>(ys, Y, LU, 32 * rb, S, LD, 32 * cb, l32, h);
        __builtin_amdgcn_sched_barrier(0);
        mm<half_t, D, false, true>(os, O, LD, 32 * rb, S, LD, 32 * cb, l32, h);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            const int p = tid + i * NT, r = p / PPR, y = p % PPR * 8;
            *reinterpret_cast<halfx8*>(S + r * LD + y) = gf[i];
        }
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
        const float up = ldexpf(1.f, ev + eg);      // of every product of two of them
        const float up12 = up * 4096.f;              // ... of Gq and Gk, which are 2^12 below theirs: sums of 128 products stay far from fp16's end
        asm volatile("" : "+v"(l32), "+v"(h));
        // one product after the other, so that no more than three are held beside dq and dk
        float pk[16], pl[16], kug = 0.f;
        const half_t *const kz = K + (32 * rb + 4 * h) * LD + 32 * cb + l32, *const qz = Q + (32 * rb + 4 * h) * LD + 32 * cb + l32;
        const float* const rz = rows + 32 * rb + 4 * h;
        auto row = [](int j) { return acc_row(j, 0); };
        f32x16 acc = zero16();
        mm<half_t, 64, false, true>(acc, Gq, LU, 32 * rb, K, LD, 32 * cb, l32, h);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float v = a.scale * (acc[j] * up12 + rz[64 + row(j)] * os[j] * up);
            dq[j] += v;
            pl[j] = (float)qz[row(j) * LD] * v;
        }
        __builtin_amdgcn_sched_barrier(0);
        acc = zero16();
        mm<half_t, 64, false, true>(acc, Gk, LU, 32 * rb, K, LD, 32 * cb, l32, h);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float kv = (float)kz[row(j) * LD], y = rz[64 + row(j)] * ys[j] * up, v = acc[j] * up12 - rz[row(j)] * y;
            pk[j] = kv * y;
            pl[j] += kv * v;
            dk[j] += v;
        }
        __builtin_amdgcn_sched_barrier(0);
        acc = zero16();
        mm<half_t, D, true, true>(acc, U, LU, 32 * rb, S, LD, 32 * cb, l32, h);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float v = rz[128 + row(j)] * acc[j] * up, kv = (float)kz[row(j) * LD];
            kug += kv * v;
            pl[j] -= kv * v;
            dk[j] += v;
        }
        __builtin_amdgcn_sched_barrier(0);
        acc = zero16();
        mm<half_t, 64, true, true>(acc, Gk, LU, 32 * rb, K, LD, 32 * cb, l32, h);
        os = zero16();
        mm<half_t, 64, true, true>(os, Gq, LU, 32 * rb, Q, LD, 32 * cb, l32, h);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float v = (acc[j] + a.scale * os[j]) * up12;
            pl[j] -= (float)kz[row(j) * LD] * v;
            dk[j] += v;
        }
        __builtin_amdgcn_sched_barrier(0);
        kug += rows[64 + 63] * sum * up;
        const float pks = sum16(pk, l32), pls = sum16(pl, l32);
        if (!(l32 & 1)) {
            kys[cb * 64 + 32 * rb + acc_row(l32 >> 1, h)] = pks;
            dls[cb * 64 + 32 * rb + acc_row(l32 >> 1, h)] = pls;
        }
#pragma unroll
        for (int z = 1; z < 64; z *= 2) kug += __shfl_xor(kug, z);
        if (lane == 0) wred[16 + wv] = kug;
        __syncthreads();
        if (wv == 0) {
            float l = 0.f, ky = 0.f, y = 0.f, all = 0.f;
#pragma unroll
            for (int i = 0; i < CB; ++i) { l += dls[i * 64 + lane]; ky += kys[i * 64 + lane]; }
#pragma unroll
            for (int i = 0; i < NWV; ++i) { y += yv[i * 64 + lane]; all += wred[16 + i]; }
#pragma unroll
            for (int z = 1; z < 64; z *= 2) {
                const float t = __shfl_down(l, z);
                if (lane + z < 64) l += t;
            }
            if (lane < left) {
                static_cast<bf16_t*>(a.dbeta)[sat + lane * a.st] = (bf16_t)(ldexpf(y, eg) - ky - (xl[lane] + xl[64 + lane]) * up);
                if (a.dlog_f) static_cast<bf16_t*>(a.dlog_f)[sat + lane * a.st] = (bf16_t)(l + all);
            }
        }
    }
    const int l32 = lane & 31, h = lane >> 5;
    bf16_t *const dqp = static_cast<bf16_t*>(a.dq) + kat, *const dkp = static_cast<bf16_t*>(a.dk) + kat;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const int r = 32 * rb + acc_row(j, h), z = 32 * cb + l32;
        if (r < left) {
            dqp[r * a.kt + z] = (bf16_t)dq[j];
            dkp[r * a.kt + z] = (bf16_t)dk[j];
        }
    }
}

template <int D> static hipError_t launch(const DeltaArgs& a, int is_bf16, hipStream_t stream) {
    const dim3 grid((unsigned)a.tiles * a.H);
    if (is_bf16) {
        static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&delta_grad16_kernel<D>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)Grad16<D>::bytes);
        if (attr != hipSuccess) return attr;
        delta_grad16_kernel<D><<<grid, dim3(Grad16<D>::NT), Grad16<D>::bytes, stream>>>(a);
    } else {
        constexpr size_t bytes = (size_t)(3 * 64 * (D + 4) + 2 * 64 * DG_LF + DELTA_ROWS * 64 + 192) * 4;
        static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&delta_grad_kernel<D>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (attr != hipSuccess) return attr;
        delta_grad_kernel<D><<<grid, dim3(256), bytes, stream>>>(a);
    }
    return hipGetLastError();
}
hipError_t launch_delta_grad(const DeltaArgs& a, int d, int is_bf16, hipStream_t stream) {
    return d == 64 ? launch<64>(a, is_bf16, stream) : launch<128>(a, is_bf16, stream);
}

}  // namespace path
