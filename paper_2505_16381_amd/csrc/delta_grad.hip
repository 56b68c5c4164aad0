// Gated delta rule: gradients of q, k, beta and log f from the states, their gradients, U and Y of a chunk, all chunks at once (delta_decl.h has the formulas).
// A workgroup takes a chunk of a key head and adds up its value heads one after the other, in registers.
#include "delta_parts.h"
#include "lds_tile.h"

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
        const float *const E = static_cast<const float*>(a.em) + u * D * 64, *const Y = static_cast<const float*>(a.ym) + u * D * 64;
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
            f32x4 X = zero, N = zero;
            if (ib <= wv)
#pragma unroll 1
                for (int z = 0; z < D; z += 16) {
                    const f32x4 uf = tr(E, 64, 16 * ib, z) * rows[16 * ib + n];
                    X = P::mma(tr(Y, 64, r0, z), uf, X);
                    N = P::mma(nat(O, LD, r0, z), uf, N);
                }
            const int i = 16 * ib + n;
            const float ih = rows[192 + i], il = rows[256 + i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = r0 + 4 * g + j;
                const float w = expf((bh[j] - ih) + (bl[j] - il));
                Gq[r * DG_LF + i] = i <= r ? a.scale * w * N[j] : 0.f;
                Gk[r * DG_LF + i] = i < r ? -be[j] * w * X[j] : 0.f;
            }
        }
        // Y.E, value indices n, n + 16, ..
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll 1
            for (int z = n; z < D; z += 16) db[j] += Y[z * 64 + r0 + 4 * g + j] * E[z * 64 + r0 + 4 * g + j];
        __syncthreads();
#pragma unroll
        for (int t = 0; t < NR; ++t) {
            f32x4 ys = zero, os = zero, ug = zero, q1 = zero, rd = zero, wr = zero;
#pragma unroll 1
            for (int z = 0; z < D; z += 16) {
                const f32x4 sf = tr(S, D, 16 * t, z);
                ys = P::mma(tr(Y, 64, r0, z), sf, ys);
                os = P::mma(nat(O, LD, r0, z), sf, os);
                ug = P::mma(tr(E, 64, r0, z) * rows[r0 + n], tr(G, D, 16 * t, z), ug);
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

// ---- bf16: 32x32 products of fp16 operands of one part (Gq and Gk: of two), over the powers of two of the scans ----
//
// A wave has 32 key indices of dq and dk, of all 64 tokens (d = 64: of 32).  E, Y and dO are in LDS for everybody; the wave's columns of S, G, K and Q pass through
// 4 KB of its own, half a state at a time, the next piece on its way in registers meanwhile: no barrier from the first product to the last but the two around Gq and Gk, and two
// workgroups on a CU.  Factors of a token (gamma, beta, rho) are multiplied into results, in 32 bits: into operands, each would be one rounding to 11 bits more, and gates above one could carry them past fp16's end.

// sums over the 32 lanes of a half-wave of each of 16 values; lane l32 gets the value l32 / 2
__device__ __forceinline__ float sum16(float (&v)[16], int l32) {
#pragma unroll
    for (int w = 8, m = 16; w >= 1; w /= 2, m /= 2) {
        const bool up = l32 & m;
#pragma unroll
        for (int j = 0; j < w; ++j) {
            float x = v[j], y = v[j + w];
            asm volatile("" : "+v"(x), "+v"(y));      // (two registers: left to itself the compiler makes it one index into sixteen, and that a chain of sixteen selections)
            v[j] = (up ? y : x) + __shfl_xor(up ? x : y, m);
        }
    }
    return v[0] + __shfl_xor(v[0], 1);
}
__device__ __forceinline__ half_t half_power(int e) { return e < -24 ? (half_t)0.f : (half_t)ldexpf(1.f, e); }

template <int D> struct Grad16 {
    static constexpr int RB = D / 64, CB = D / 32;                     // blocks of 32 tokens of a wave, of 32 key indices of a head
    static constexpr int TOK = 64 * D * 2, G2 = 64 * 64 * 2;            // bytes of a tokens' matrix, of Gq
    static constexpr int E = 0, Y = TOK, O = 2 * TOK, SLOT = O + (TOK > 2 * G2 ? TOK : 2 * G2), ROWS = SLOT + 4 * 4096, RED = ROWS + DELTA_ROWS * 256;
    static constexpr int BYTES = RED + (4 * 64 + CB * 64 + 16) * 4;
    static_assert(2 * G2 <= O - E, "the second parts of Gq and Gk lie in E's and Y's place");
};

// ---- bf16: 32x32x16 products of fp16 operands; E, Y, dO (then Gq and Gk in their place) in LDS, S and G by way of 4 KB of a wave's own ----
//
// A wave has 32 key indices; two workgroups share a CU, so that one's loads stand beside the other's products.  Bound by memory, and by the chain of a chunk's phases: d = 128, 64 heads of 8192 tokens 484 to 529 us from run to run, 3.0 TB/s and more of its own traffic
// (1.61 GB: S, G, E, Y, K, Q, dO in, dq, dk, dv out); 16 value heads of 8 key heads over 15000 tokens, whose groups of two add up in registers (97 of them spilled, 384 bytes a lane), 352 us.  With Gq and Gk as single
// numbers 407 to 450 us, in groups 292.  Before that: with S and G whole in LDS (one workgroup per CU) 1098 us, by way of a wave's own 4 KB 561, with row sums in registers that no index selects and gradients out by whole
// pieces 429.
template <int D, bool GROUP>
__global__ __launch_bounds__(256, 2) void delta_grad16_kernel(DeltaArgs a) {
    typedef Grad16<D> C;
    typedef TurnedLane<64> Lane;      // of E, Y, Gq, Gk
    constexpr int RB = C::RB, CB = C::CB, NP = 64 * D / 8 / 256;      // 16-byte pieces of a tokens' matrix per thread
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    float* const rows = reinterpret_cast<float*>(smem + C::ROWS);
    float *const dbs = reinterpret_cast<float*>(smem + C::RED), *const dls = dbs + 256, *const kus = dls + CB * 64, *const mosts = kus + 4;      // [wave][64], [column block][64], [wave], [block of pairs]
    int tid = threadIdx.x, lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tile = __builtin_amdgcn_readfirstlane(blockIdx.x / a.H), hk = blockIdx.x - tile * a.H;
    int s, c;
    DeltaSeq sq;
    if (!delta_tile(a, tile, lane, s, c, sq)) return;
    const int t0 = c * CHUNK, left = sq.len - t0;
    const int cb = wv % CB, rb0 = RB == 2 ? 0 : wv / CB;      // the wave's column block, its first block of tokens
    const long long kat = delta_at(a, sq, s, a.ks, a.kt) + hk * a.kh + t0 * a.kt;
    const bf16_t *const kp = static_cast<const bf16_t*>(a.k) + kat + 32 * cb, *const qp = static_cast<const bf16_t*>(a.q) + kat + 32 * cb;
    half_t* const slot = reinterpret_cast<half_t*>(smem + C::SLOT + wv * 4096);      // [64][32]
    f32x16 dq[RB], dk[RB];
    if (GROUP)
#pragma unroll
        for (int b = 0; b < RB; ++b) dq[b] = dk[b] = zero16();
    // the wave's 32 columns of 64 rows, from fragments of 16 rows (delta_scan.hip): 16 bytes a lane, row lane % 16 + 16 i
    auto slice_rows = [&](const half_t* x, halfx8 (&f)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = *reinterpret_cast<const halfx8*>(x + i * CB * 512 + lane * 8);
    };
    auto slice_tokens = [&](const bf16_t* x, bf16x8 (&f)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = lane / 4 + 16 * i;
#pragma unroll
            for (int e = 0; e < 8; ++e) f[i][e] = (bf16_t)0.f;
            if (r < left) f[i] = *reinterpret_cast<const bf16x8*>(x + r * a.kt + lane % 4 * 8);
        }
    };
    auto operands = [&](const bf16x8 (&x)[4], float w, halfx8 (&f)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) f[i][e] = (half_t)((float)x[i][e] * w);
    };
    // the wave's block of a gradient, by whole pieces: through its own LDS
    auto out_rows = [&](void* base, const f32x16 (&x)[RB]) {
        bf16_t* const to = reinterpret_cast<bf16_t*>(slot);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int j = 0; j < 16; ++j) to[(32 * b + acc_row(j, lane >> 5)) * 32 + (lane & 31)] = (bf16_t)x[b][j];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 2 * RB; ++i) {
            const int r = lane / 4 + 16 * i;
            const bf16x8 f = *reinterpret_cast<const bf16x8*>(to + r * 32 + lane % 4 * 8);
            if (32 * rb0 + r < left) *reinterpret_cast<bf16x8*>(static_cast<bf16_t*>(base) + kat + (32 * rb0 + r) * a.kt + 32 * cb + lane % 4 * 8) = f;
        }
    };
    auto to_slot = [&](const halfx8 (&f)[4]) {
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<halfx8*>(slot + (lane / 4 + 16 * i) * 32 + lane % 4 * 8) = f[i];
        __builtin_amdgcn_wave_barrier();
    };
    auto frags_to_slot = [&](const halfx8 (&f)[4]) {
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<halfx8*>(slot + ((lane & 15) + 16 * i) * 32 + (lane >> 4) * 8) = f[i];
        __builtin_amdgcn_wave_barrier();
    };
#pragma unroll 1
    for (int x = 0; x < (GROUP ? a.G : 1); ++x) {
        const int hv = hk * a.G + x;
        // (the lane's place, made anew: addresses of all products kept across the loop over heads would not fit the registers)
        if (GROUP) asm volatile("" : "+v"(tid), "+v"(lane));
        const int l32 = lane & 31, h = lane >> 5;
        const size_t u = (size_t)tile * a.V + hv;
        const long long vat = delta_at(a, sq, s, a.vs, a.vt) + hv * a.vh + t0 * a.vt, sat = delta_at(a, sq, s, a.ss, a.st) + hv * a.sh + t0 * a.st;
        const half_t *const sg = static_cast<const half_t*>(a.sm) + u * D * D + 512 * cb, *const gg = static_cast<const half_t*>(a.gm) + u * D * D + 512 * cb;
        const half_t *const eg = static_cast<const half_t*>(a.em) + u * D * 64, *const yg = static_cast<const half_t*>(a.ym) + u * D * 64;
        const int *const vex = a.vex + ((size_t)s * a.V + hv) * 8, *const gex = a.gex + ((size_t)s * a.V + hv) * 8;
        int ev = vex[0], eq = gex[0];      // the largest exponents: of S and E, of G, Y and dO
#pragma unroll
        for (int b = 1; b < D / 16; ++b) {
            ev = vex[b] > ev ? vex[b] : ev;
            eq = gex[b] > eq ? gex[b] : eq;
        }
        __syncthreads();      // (the head before has been read out)
        halfx8 sf[4], gf[4];
        {
            halfx8 ef[NP], yf[NP];
            bf16x8 of[NP];
            const int y = 32 * (wv & 1) + 8 * (lane >> 4);      // the first of the eight tokens of the thread's pieces of E and Y
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int p = tid + i * 256, r = p / (D / 8);      // of dO; E and Y: fragments
                ef[i] = *reinterpret_cast<const halfx8*>(eg + p * 8);
                yf[i] = *reinterpret_cast<const halfx8*>(yg + p * 8);
#pragma unroll
                for (int e = 0; e < 8; ++e) of[i][e] = (bf16_t)0.f;
                if (r < left) of[i] = *reinterpret_cast<const bf16x8*>(static_cast<const bf16_t*>(a.d_o) + vat + r * a.vt + p % (D / 8) * 8);
            }
            slice_rows(sg, sf);
            slice_rows(gg, gf);
            for (int i = tid; i < DELTA_ROWS * 64; i += 256) rows[i] = a.rows[u * DELTA_ROWS * 64 + i];
            const float wo = delta_power(-eq);
            float db[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int p = tid + i * 256, vt = (wv >> 1) + 2 * i, r = 16 * vt + (lane & 15), ro = p / (D / 8), xo = p % (D / 8) * 8;
                const halfx8 e1 = ef[i] * half_power(vex[vt] - ev), y1 = yf[i] * half_power(gex[vt] - eq);      // (Y goes to LDS over its own columns' power: dv is made of it)
#pragma unroll
                for (int e = 0; e < 8; ++e) db[e] += (float)e1[e] * (float)y1[e];
                *reinterpret_cast<halfx8*>(smem + C::E + 2 * TurnedTile<64>::at(r, y)) = e1;
                *reinterpret_cast<halfx8*>(smem + C::Y + 2 * TurnedTile<64>::at(r, y)) = yf[i];
                halfx8 o1;
#pragma unroll
                for (int e = 0; e < 8; ++e) o1[e] = (half_t)((float)of[i][e] * wo);
                *reinterpret_cast<halfx8*>(smem + C::O + 2 * TurnedTile<D>::at(ro, xo)) = o1;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int z = 1; z < 16; z *= 2) db[e] += __shfl_xor(db[e], z);
            if ((lane & 15) == 0)
#pragma unroll
                for (int e = 0; e < 8; ++e) dbs[wv * 64 + y + e] = db[e];
        }
        __syncthreads();

        const Lane at(lane);
        const TurnedLane<D> ato(lane);
        auto u_frag = [&](int mat, int b, int sl) {      // tokens 32 b .. along the lanes, value indices 16 sl .. as the contraction
            typedef short v4s __attribute__((ext_vector_type(4)));
            union { v4s v[2]; halfx8 f; } w;
            w.v[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(smem + mat + at.tr_at(16 * sl, 32 * b, 0)));
            w.v[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(smem + mat + at.tr_at(16 * sl, 32 * b, 1)));
            return w.f;
        };
        auto o_frag = [&](int b, int sl) { return *reinterpret_cast<const halfx8*>(smem + C::O + ato.nat_at(32 * b, 16 * sl)); };
        auto slot_frag = [&](int sl) { return ld_frag_tr<half_t>(slot, 32, 16 * sl, 0, l32, h); };
        f32x16 q1[RB], rd[RB], wr[RB];
        float sum = 0.f;      // <S, G>, over 2^(ev + eq)
        {
            float bt[RB];      // beta of the lane's tokens
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                bt[b] = rows[32 * (rb0 + b) + l32];
                q1[b] = rd[b] = wr[b] = zero16();
            }
            bf16_t* const dvp = static_cast<bf16_t*>(a.dv) + vat;
#pragma unroll 1
            for (int half = 0; half < D / 64; ++half) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sf[i] = sf[i] * half_power(vex[4 * half + i] - ev);
                    gf[i] = gf[i] * half_power(gex[4 * half + i] - eq);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum += (float)sf[i][e] * (float)gf[i][e];
                }
                frags_to_slot(sf);
                if (half + 1 < D / 64) slice_rows(sg + (size_t)64 * D, sf);
#pragma unroll
                for (int sl = 0; sl < 4; ++sl) {
                    const halfx8 f = slot_frag(sl);
                    const int ey = gex[4 * half + sl];      // of these 16 value indices
                    const half_t hy = half_power(ey - eq);
                    const float wdv = delta_power(ey);
#pragma unroll
                    for (int b = 0; b < RB; ++b) {
                        const halfx8 y = u_frag(C::Y, rb0 + b, 4 * half + sl);
                        q1[b] = Tr<half_t>::mma(o_frag(rb0 + b, 4 * half + sl), f, q1[b]);
                        rd[b] = Tr<half_t>::mma(y * hy, f, rd[b]);
                        if ((RB == 2 ? sl : sl & 1) == cb) {      // dv = beta Y: 8 value indices of the lane's token; the waves take turns
                            const int r = 32 * (rb0 + b) + l32;
                            bf16x8 v;
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] = (bf16_t)((float)y[e] * (bt[b] * wdv));
                            if (r < left) *reinterpret_cast<bf16x8*>(dvp + r * a.vt + 16 * (4 * half + sl) + 8 * h) = v;
                        }
                    }
                }
                frags_to_slot(gf);
                if (half + 1 < D / 64) slice_rows(gg + (size_t)64 * D, gf);
#pragma unroll
                for (int sl = 0; sl < 4; ++sl) {
                    const halfx8 f = slot_frag(sl);
#pragma unroll
                    for (int b = 0; b < RB; ++b) wr[b] = Tr<half_t>::mma(u_frag(C::E, rb0 + b, 4 * half + sl), f, wr[b]);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 kr[4];
        slice_tokens(kp, kr);
        // X and N of the lower 32x32 blocks.  Gq and Gk are sums of two fp16 numbers: in dlog_f they add up, times products of keys, over pairs of tokens, and over keys alike those sums cancel where independent
        // roundings of the pairs do not (single ones left dlog_f off by 6e-3 of its norm at products of 0.95).  They are over a power of two of their own, from the largest of
        // both: what they are made of may have been walked again with 2^16 times the room, and lie that much lower, or have grown.  The second parts take E's and Y's place.  A wave's first block waits in the 4 KB of its own.
        f32x16 pairs;
        f32x4* const parked = reinterpret_cast<f32x4*>(slot);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int job = wv + 4 * n, b = job % 3, br = b ? 1 : 0, bi = b == 2 ? 1 : 0;
            if (job < 6) {
                f32x16 acc = zero16();
#pragma unroll
                for (int sl = 0; sl < D / 16; ++sl) {
                    const halfx8 f = u_frag(C::E, bi, sl);
                    acc = Tr<half_t>::mma(job < 3 ? u_frag(C::Y, br, sl) * half_power(gex[sl] - eq) : o_frag(br, sl), f, acc);
                }
                const int i = 32 * bi + l32;
                const float ih = rows[192 + i], il = rows[256 + i], ib = rows[i];
                float top = 0.f;
#pragma unroll
                for (int j4 = 0; j4 < 16; j4 += 4) {
                    const int r0 = 32 * br + acc_row(j4, h);
                    const f32x4 rh = *reinterpret_cast<const f32x4*>(rows + 192 + r0), rl = *reinterpret_cast<const f32x4*>(rows + 256 + r0), rb = *reinterpret_cast<const f32x4*>(rows + r0);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        // (a power of two: its rounding and that of the exponent, 1e-5, are nothing beside those of E and Y)
                        const float w = ib * __builtin_amdgcn_exp2f(((rh[j] - ih) + (rl[j] - il)) * 1.44269504088896340736f);
                        pairs[j4 + j] = job < 3 ? (i < r0 + j ? -rb[j] * w * acc[j4 + j] : 0.f) : (i <= r0 + j ? w * acc[j4 + j] : 0.f);
                        top = fmaxf(top, delta_finite(pairs[j4 + j]));
                    }
                }
#pragma unroll
                for (int z = 1; z < 64; z *= 2) top = fmaxf(top, __shfl_xor(top, z));
                if (lane == 0) mosts[job] = top;
                if (n == 0)
#pragma unroll
                    for (int p = 0; p < 4; ++p) parked[p * 64 + lane] = f32x4{pairs[4 * p], pairs[4 * p + 1], pairs[4 * p + 2], pairs[4 * p + 3]};
            }
        }
        __syncthreads();      // (E, Y and dO have been read: Gq and Gk take their places)
        // the largest between 2^13 and 2^14: sums of two fp16 numbers are right to 2^-38 of it and more
        float most = mosts[0];
#pragma unroll
        for (int i = 1; i < 6; ++i) most = fmaxf(most, mosts[i]);
        const int above = most > 0.f ? 8 - delta_exponent(most) : 0, raised = __builtin_amdgcn_readfirstlane(above < -40 ? -40 : above > 40 ? 40 : above);
#pragma unroll
        for (int n = 1; n >= 0; --n) {
            const int job = wv + 4 * n, b = job % 3, br = b ? 1 : 0, bi = b == 2 ? 1 : 0;
            if (n == 0)
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const f32x4 x = parked[p * 64 + lane];
#pragma unroll
                    for (int e = 0; e < 4; ++e) pairs[4 * p + e] = x[e];
                }
            if (job < 6) {
                half_t* const to = reinterpret_cast<half_t*>(smem + C::O + (job < 3 ? C::G2 : 0));
                half_t* const to2 = reinterpret_cast<half_t*>(smem + C::E + (job < 3 ? C::G2 : 0));
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int i = TurnedTile<64>::at(32 * br + acc_row(j, h), 32 * bi + l32);
                    const float y = ldexpf(pairs[j], raised);
                    const half_t y1 = (half_t)y;
                    to[i] = y1;
                    to2[i] = (half_t)(y - (float)y1);
                }
                if (b == 1)      // the upper block
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const int i = TurnedTile<64>::at(acc_row(j, h), 32 + l32);
                        to[i] = to2[i] = (half_t)0.f;
                    }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        halfx8 kf[4];
        operands(kr, 1.f, kf);
        to_slot(kf);
        slice_tokens(qp, kr);
        __syncthreads();
        const float up = ldexpf(1.f, ev + eq), upg = ldexpf(1.f, ev + eq - raised), wg = delta_power(raised);      // of every product of two of them, of Gq and Gk
        auto nat = [&](int mat, int b, int sl) { return *reinterpret_cast<const halfx8*>(smem + mat + at.nat_at(32 * b, 16 * sl)); };
        float kug = 0.f;
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int j4 = 0; j4 < 16; j4 += 4) {
                const int r0 = 32 * (rb0 + b) + acc_row(j4, h);
                const f32x4 be = *reinterpret_cast<const f32x4*>(rows + r0), ga = *reinterpret_cast<const f32x4*>(rows + 64 + r0), rh = *reinterpret_cast<const f32x4*>(rows + 128 + r0);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = j4 + e;
                    wr[b][j] *= rh[e] * be[e];
                    kug += (float)slot[(r0 + e) * 32 + l32] * wr[b][j];
                    q1[b][j] *= wg * ga[e];
                    rd[b][j] *= -wg * ga[e] * be[e];
                    wr[b][j] *= wg;
                }
            }
        kug = (kug + (rb0 == 0 ? rows[64 + 63] * sum : 0.f)) * up;
#pragma unroll
        for (int sl = 0; sl < 4; ++sl) {
            const halfx8 f = slot_frag(sl);
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                const int br = rb0 + b;
                // (Gq and Gk are lower triangular: 32 tokens are before or behind the others)
                if (br == 1 || sl < 2) {
#pragma unroll
                    for (const int part : {C::E, C::O}) {
                        q1[b] = Tr<half_t>::mma(nat(part, br, sl), f, q1[b]);
                        rd[b] = Tr<half_t>::mma(nat(part + C::G2, br, sl), f, rd[b]);
                    }
                }
                if (br == 0 || sl >= 2)
#pragma unroll
                    for (const int part : {C::E, C::O}) wr[b] = Tr<half_t>::mma(u_frag(part + C::G2, br, sl), f, wr[b]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        // k.dk before Q takes K's place; then q.dq
        halfx8 kl[RB][2];
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int j = 0; j < 16; ++j) kl[b][j / 8][j % 8] = slot[(32 * (rb0 + b) + acc_row(j, h)) * 32 + l32];
        operands(kr, a.scale, kf);
        to_slot(kf);
#pragma unroll
        for (int sl = 0; sl < 4; ++sl) {
            const halfx8 f = slot_frag(sl);
#pragma unroll
            for (int b = 0; b < RB; ++b)
                if (rb0 + b == 0 || sl >= 2)
#pragma unroll
                    for (const int part : {C::E, C::O}) wr[b] = Tr<half_t>::mma(u_frag(part, rb0 + b, sl), f, wr[b]);
        }
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            float pl[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int r = 32 * (rb0 + b) + acc_row(j, h);
                const float d1 = q1[b][j] * upg, d2 = rd[b][j] * upg, d3 = wr[b][j] * upg;      // (dq without scale: so is Q with it)
                pl[j] = (float)slot[r * 32 + l32] * d1 + (float)kl[b][j / 8][j % 8] * (d2 - d3);
                q1[b][j] = a.scale * d1;
                rd[b][j] = d2 + d3;
                if (GROUP) {
                    dq[b][j] += q1[b][j];
                    dk[b][j] += rd[b][j];
                }
            }
            const float y = sum16(pl, l32);
            if (!(l32 & 1)) dls[cb * 64 + 32 * (rb0 + b) + acc_row(l32 >> 1, h)] = y;
        }
#pragma unroll
        for (int z = 1; z < 64; z *= 2) kug += __shfl_xor(kug, z);
        if (lane == 0) kus[wv] = kug;
        __syncthreads();
        if (wv == 0) {
            float l = 0.f;
#pragma unroll
            for (int i = 0; i < CB; ++i) l += dls[i * 64 + lane];
#pragma unroll
            for (int z = 1; z < 64; z *= 2) {
                const float y = __shfl_down(l, z);
                if (lane + z < 64) l += y;
            }
            if (lane < left) {
                static_cast<bf16_t*>(a.dbeta)[sat + lane * a.st] = (bf16_t)((dbs[(lane >> 5) * 64 + lane] + dbs[((lane >> 5) + 2) * 64 + lane]) * up);      // (of the two waves that have the token's half)
                if (a.dlog_f) static_cast<bf16_t*>(a.dlog_f)[sat + lane * a.st] = (bf16_t)(l + ((kus[0] + kus[1]) + (kus[2] + kus[3])));
            }
        }
        if (!GROUP) {
            out_rows(a.dq, q1);
            out_rows(a.dk, rd);
        } else if (x + 1 == a.G) {
            out_rows(a.dq, dq);
            out_rows(a.dk, dk);
        }
    }
}

template <int D, bool GROUP> static hipError_t launch16(const DeltaArgs& a, hipStream_t stream) {
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&delta_grad16_kernel<D, GROUP>), hipFuncAttributeMaxDynamicSharedMemorySize, Grad16<D>::BYTES);
    if (attr != hipSuccess) return attr;
    delta_grad16_kernel<D, GROUP><<<dim3((unsigned)a.tiles * a.H), dim3(256), Grad16<D>::BYTES, stream>>>(a);
    return hipGetLastError();
}
template <int D> static hipError_t launch(const DeltaArgs& a, int is_bf16, hipStream_t stream) {
    const dim3 grid((unsigned)a.tiles * a.H);
    if (is_bf16) {
        return a.G > 1 ? launch16<D, true>(a, stream) : launch16<D, false>(a, stream);
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
