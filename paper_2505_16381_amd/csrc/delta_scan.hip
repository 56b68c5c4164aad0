// Gated delta rule: the states, chunk after chunk, and backwards their gradients (delta_decl.h has the formulas).
//
// A workgroup of four waves has CT * 16 columns (value indices) of a head's state, which stays in registers: each wave a quarter of its rows (key indices), and of a chunk's
// products with it the 16 tokens of one result tile.  What a wave needs of K, Q, A and M nobody else needs, so it comes from memory straight into its
// registers, a chunk ahead; what all need -- the state, the predictions' errors, U -- is exchanged through LDS as operands, split once.  Three barriers a chunk.
#include "delta_parts.h"

namespace path {

enum { DELTA_O = 0, DELTA_KEEP = 1, DELTA_BACK = 2 };      // forward; forward that keeps what the backward needs; backwards

template <typename T, int D, int NP, int CT, int MODE>
struct ScanLds {
    typedef DeltaOps<T> P;
    static constexpr int NS = D / P::SL, CS = 64 / P::SL;                      // slabs of the state's rows, of a chunk
    static constexpr int TW = D / 64;                                          // state tiles of a wave
    static constexpr int SW = sizeof(T) == 2 ? 32 : 16 * TW, SROW = sizeof(T) == 2 ? 64 : (SW + 4) * 4;      // a wave's columns of K: elements, bytes of a row in LDS
    static constexpr int SLICE = 64 * SROW, NSL = MODE == DELTA_BACK ? 2 : 1;
    static constexpr int S = 0, Y = S + NS * NP * CT * 1024, U = Y + CS * NP * CT * 1024, V = U + CS * NP * CT * 1024, O = V + CS * NP * CT * 1024;
    static constexpr int X = O + (MODE == DELTA_BACK ? CS * CT * 1024 : 0), KT = X + 256, BYTES = KT + 4 * NSL * SLICE;
};

// largest |x| of a wave's values; the exponent that leaves fp16 numbers below 2^11
__device__ __forceinline__ float delta_most(float m) {
#pragma unroll
    for (int i = 1; i < 64; i *= 2) m = fmaxf(m, __shfl_xor(m, i));
    return m;
}
__device__ __forceinline__ int delta_exponent(float m) {
    const int e = (int)(__float_as_uint(m) >> 23) - 127 - 10;
    return e < -126 ? -126 : e;
}

template <typename T, int D, int NP, int CT, int MODE>
__global__ __launch_bounds__(256, CT == 2 ? 1 : 2) void delta_scan_kernel(DeltaArgs a) {
    typedef DeltaOps<T> P;
    typedef typename P::Frag Frag;
    typedef ScanLds<T, D, NP, CT, MODE> L;
    constexpr int NS = L::NS, CS = L::CS, TW = L::TW;
    constexpr bool BACK = MODE == DELTA_BACK;
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    int unit, part;
    if (!xcd_deal(blockIdx.x >> 3, blockIdx.x & 7, D / 16 / CT, a.nseq * a.V, unit, part)) return;
    const int s = __builtin_amdgcn_readfirstlane(unit / a.V), hv = unit - s * a.V, hk = __builtin_amdgcn_readfirstlane(hv / a.G);
    const DeltaSeq sq = delta_seq(a, s);
    const int len = __builtin_amdgcn_readfirstlane(sq.len), tile0 = __builtin_amdgcn_readfirstlane(sq.tile0);
    if (a.slots && len <= a.few) return;
    const int NC = (len + CHUNK - 1) / CHUNK;
    const int col = 16 * part * CT + n;      // the lane's value index (and + 16)

    // the first state: of a pool's slot, given, or zeros
    f32x4 S[TW][CT];
    const size_t head = ((size_t)s * a.V + hv) * D * D;
    const float* from = nullptr;
    float* to = nullptr;
    if (BACK) {
        from = a.d_state ? a.d_state + head : nullptr;
        to = a.d_state_in ? a.d_state_in + head : nullptr;
    } else if (a.slots) {
        const int slot = a.slots[s];
        if (slot >= 0 && slot < a.num_slots) {
            to = a.states + ((size_t)slot * a.V + hv) * D * D;
            if (a.cached[s] > 0) from = to;
        }
    } else {
        from = a.state_in ? a.state_in + head : nullptr;
        to = a.state_out ? a.state_out + head : nullptr;
    }
#pragma unroll
    for (int t = 0; t < TW; ++t)
#pragma unroll
        for (int x = 0; x < CT; ++x)
#pragma unroll
            for (int j = 0; j < 4; ++j) S[t][x][j] = from ? from[(size_t)P::row(TW * wv + t, 4 * g + j) * D + col + 16 * x] : 0.f;

    // an exchange area's fragment, and one tile of a slab as operands into it
    auto frag = [&](int area, int sl, int x) {
        DeltaParts<T, NP> f;
#pragma unroll
        for (int p = 0; p < NP; ++p) f.p[p] = *reinterpret_cast<const Frag*>(smem + area + ((sl * CT + x) * NP + p) * 1024 + lane * 16);
        return f;
    };
    auto put = [&](int area, int tile, int x, const f32x4& v) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<f32x4*>(smem + area + (tile * CT + x) * 1024 + lane * 16) = v;
        } else {
            DeltaSplit4<NP> r(v);
#pragma unroll
            for (int p = 0; p < NP; ++p)
                *reinterpret_cast<uint2*>(smem + area + (((tile >> 1) * CT + x) * NP + p) * 1024 + lane * 16 + (tile & 1) * 8) = r.p[p];
        }
    };

    // Addresses: a chunk's place in scalar registers, the lane's in 32 bits of bytes, made anew only where a chunk has fewer than 64 tokens: rows behind the sequence's end are
    // its last one again (their beta is 0).
    constexpr int ES = sizeof(T), PPR = L::SW * ES / 16, NK = PPR;      // 16-byte pieces of a slice's row; of a slice per lane
    const char* const kb = static_cast<const char*>(a.k) + (delta_at(a, sq, s, a.ks, a.kt) + hk * a.kh) * ES;
    const char* const qb = static_cast<const char*>(a.q) + (delta_at(a, sq, s, a.ks, a.kt) + hk * a.kh) * ES;
    const long long vat = (delta_at(a, sq, s, a.vs, a.vt) + hv * a.vh + 16 * part * CT) * ES;
    const char* const vb = static_cast<const char*>(BACK ? a.d_o : a.v) + vat;
    char* const ob = static_cast<char*>(BACK ? a.dv : a.o) + vat;
    const long long kstep = a.kt * ES * CHUNK, vstep = a.vt * ES * CHUNK;
    unsigned row_at, slice_at[NK], value_at[4];
    auto place = [&](int c) {
        const int last = len - 1 - c * CHUNK;
        const unsigned kt = (unsigned)a.kt * ES, vt = (unsigned)a.vt * ES;
        auto held = [&](int r) { return (unsigned)(r < last ? r : last); };
        row_at = held(P::row(wv, n)) * kt + 16 * g;
        const int c0 = sizeof(T) == 2 ? 32 * (TW * wv >> 1) : 16 * TW * wv;
#pragma unroll
        for (int i = 0; i < NK; ++i) slice_at[i] = held((i * 64 + lane) / PPR) * kt + c0 * ES + (lane % PPR) * 16;
#pragma unroll
        for (int j = 0; j < 4; ++j) value_at[j] = held(P::row(wv, 4 * g + j)) * vt + n * ES;
    };
    auto partial = [&](int c) { return len - c * CHUNK < CHUNK; };

    // What a chunk brings, loaded again as soon as it has been used.
    Frag K[NS], Q[BACK ? 1 : NS], kt[L::NSL][NK];
    DeltaParts<T, NP> A[CS], M[CS];
    T v[CT][4];
    f32x4 be, ga4, rh;
    float g63;
    typedef const __attribute__((address_space(1))) Frag GlobalFrag;
    auto load_rows = [&](const char* base, int c, Frag* f) {
        const GlobalBytes p = scalar_base(base + c * kstep, row_at);
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) f[sl] = *(GlobalFrag*)(p + sl * P::SL * ES);
    };
    auto load_slice = [&](const char* base, int c, Frag* f) {      // all rows of the wave's columns
#pragma unroll
        for (int i = 0; i < NK; ++i) f[i] = *(GlobalFrag*)scalar_base(base + c * kstep, slice_at[i]);
    };
    auto store_slice = [&](const Frag* f, int at) {
#pragma unroll
        for (int i = 0; i < NK; ++i) *reinterpret_cast<Frag*>(smem + at + (i * 64 + lane) / PPR * L::SROW + (lane % PPR) * 16) = f[i];
    };
    auto used = [&](int sl) { return BACK ? P::up(wv, sl) : P::low(wv, sl); };
    auto load_tri = [&](const void* base, int c, DeltaParts<T, NP>* f) {      // (without branches: a slab that is not used is the wave's first or last one again)
        const char* const p = static_cast<const char*>(base) + ((size_t)(tile0 + c) * a.V + hv) * NP * P::NLOW * 1024;
#pragma unroll
        for (int sl = 0; sl < CS; ++sl) {
            const int at = BACK ? P::up_at(wv, used(sl) ? sl : CS - 1) : P::low_at(wv, used(sl) ? sl : 0);
#pragma unroll
            for (int z = 0; z < NP; ++z) f[sl].p[z] = *(GlobalFrag*)scalar_base(p + (z * P::NLOW + at) * 1024, lane * 16);
        }
    };
    auto load_values = [&](int c) {      // the lane's tokens and columns of V (backwards: dO)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int x = 0; x < CT; ++x) v[x][j] = *(const __attribute__((address_space(1))) T*)(scalar_base(vb + c * vstep, value_at[j]) + 16 * x * ES);
    };
    auto load_numbers = [&](int c) {
        const float* const p = a.rows + ((size_t)(tile0 + c) * a.V + hv) * DELTA_ROWS * 64;
        typedef const __attribute__((address_space(1))) f32x4 Global4;
        const GlobalBytes r = scalar_base(p, P::row(wv, 4 * g) * 4);
        be = *(Global4*)r;
        ga4 = *(Global4*)(r + 256);
        rh = *(Global4*)(r + 512);
        g63 = p[64 + 63];
    };
    unsigned out_at[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) out_at[j] = P::row(wv, 4 * g + j) * ((unsigned)a.vt * ES) + n * ES;
    const void *const ga = BACK ? a.at : a.a, *const gm = BACK ? a.mt : a.m;
    const int slice = L::KT + wv * L::NSL * L::SLICE;
    // state tiles += (the wave's columns of K or Q)^T y
    auto into_state = [&](int at, const DeltaParts<T, NP> (&y)[CS][CT]) {
        if constexpr (sizeof(T) == 2) {
            const unsigned base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)(smem + at) + (8 * g + (n >> 2)) * 64 + (n & 3) * 16;
            bf16x8 f[2][2];
            delta_ld_tr<32>(base, f);
#pragma unroll
            for (int sl = 0; sl < 2; ++sl)
#pragma unroll
                for (int t = 0; t < TW; ++t)
#pragma unroll
                    for (int x = 0; x < CT; ++x) {
                        DeltaParts<T, 1> k;
                        k.p[0] = TW == 2 ? f[t][sl] : (wv & 1) ? f[1][sl] : f[0][sl];
                        S[t][x] = delta_mma(k, y[sl][x], S[t][x]);
                    }
        } else {
#pragma unroll
            for (int sl = 0; sl < CS; ++sl)
#pragma unroll
                for (int t = 0; t < TW; ++t) {
                    DeltaParts<T, 1> k;
#pragma unroll
                    for (int e = 0; e < 4; ++e) k.p[0][e] = *reinterpret_cast<const float*>(smem + at + (16 * sl + 4 * g + e) * L::SROW + (16 * t + n) * 4);
#pragma unroll
                    for (int x = 0; x < CT; ++x) S[t][x] = delta_mma(k, y[sl][x], S[t][x]);
                }
        }
    };
    // an exchange area's slabs, requested together: left to itself the compiler waits for each on its own
    auto frags = [&](int area, DeltaParts<T, NP> (&f)[CS][CT]) {
#pragma unroll
        for (int sl = 0; sl < CS; ++sl)
#pragma unroll
            for (int x = 0; x < CT; ++x) f[sl][x] = frag(area, sl, x);
    };
    float* const xs = reinterpret_cast<float*>(smem + L::X);      // largest values: [2][CT][wave]
    auto put_state = [&]() {
#pragma unroll
        for (int x = 0; x < CT; ++x) {
            float m = 0.f;
#pragma unroll
            for (int t = 0; t < TW; ++t) {
                put(L::S, TW * wv + t, x, S[t][x]);
                if (MODE != DELTA_O && sizeof(T) == 2)
#pragma unroll
                    for (int j = 0; j < 4; ++j) m = fmaxf(m, fabsf(S[t][x][j]));
            }
            if (MODE != DELTA_O && sizeof(T) == 2) {
                m = delta_most(m);
                if (lane == 0) xs[x * 4 + wv] = m;
            }
        }
    };
    auto put_most = [&](const f32x4* w) {      // of a token tile
        if (MODE != DELTA_O && sizeof(T) == 2)
#pragma unroll
            for (int x = 0; x < CT; ++x) {
                const float m = delta_most(fmaxf(fmaxf(fabsf(w[x][0]), fabsf(w[x][1])), fmaxf(fabsf(w[x][2]), fabsf(w[x][3]))));
                if (lane == 0) xs[16 + x * 4 + wv] = m;
            }
    };
    // a tile to memory for the chunk's gradients, the lane's row of the transposed matrix: fp32, or fp16 over a power of two of the 16 columns
    auto keep = [&](void* out, int which, int at, int x, size_t u, int ld, int tile, const f32x4& w) {
        const size_t row = (u * D + col + 16 * x) * ld + P::row(tile, 4 * g);
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<f32x4*>(static_cast<float*>(out) + row) = w;
        } else {
            const f32x4 m = *reinterpret_cast<const f32x4*>(xs + at + x * 4);
            const int ex = delta_exponent(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])));
            if (tid == 0) a.ex[u * 32 + which * 8 + part * CT + x] = ex;
            halfx4 h;
#pragma unroll
            for (int j = 0; j < 4; ++j) h[j] = (half_t)ldexpf(w[j], -ex);
            *reinterpret_cast<halfx4*>(static_cast<half_t*>(out) + row) = h;
        }
    };

    const int step = BACK ? -1 : 1;
    int c = BACK ? NC - 1 : 0;
    if (NC > 0) {
        place(c);
        load_rows(kb, c, K);
        if (!BACK) load_rows(qb, c, Q);
        load_numbers(c);
        load_values(c);
        load_tri(ga, c, A);
        load_tri(gm, c, M);
        load_slice(kb, c, kt[0]);
        if (BACK) load_slice(qb, c, kt[L::NSL - 1]);
    }
    put_state();
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < NC; ++i, c += step) {
        const int next = i + 1 < NC ? c + step : c;      // (the last chunk's loads are its own again)
        const size_t u = (size_t)(tile0 + c) * a.V + hv;
        f32x4 V[CT], ys[CT], os[CT];
#pragma unroll
        for (int x = 0; x < CT; ++x)
#pragma unroll
            for (int j = 0; j < 4; ++j) V[x][j] = c * CHUNK + P::row(wv, 4 * g + j) < len ? (float)v[x][j] : 0.f;
        if (partial(next) != partial(c)) place(next);
        load_values(next);
        store_slice(kt[0], slice);
        if (BACK) {
            store_slice(kt[L::NSL - 1], slice + L::SLICE);
#pragma unroll
            for (int x = 0; x < CT; ++x) {      // dO is an operand as it is
                if constexpr (sizeof(T) == 4) {
                    *reinterpret_cast<f32x4*>(smem + L::O + (wv * CT + x) * 1024 + lane * 16) = V[x];
                } else {
                    bf16x4 b;
#pragma unroll
                    for (int j = 0; j < 4; ++j) b[j] = (bf16_t)V[x][j];
                    *reinterpret_cast<bf16x4*>(smem + L::O + ((wv >> 1) * CT + x) * 1024 + lane * 16 + (wv & 1) * 8) = b;
                }
            }
        }
        load_slice(kb, next, kt[0]);
        if (BACK) load_slice(qb, next, kt[L::NSL - 1]);
        lds_barrier();

        // K S and Q S of the wave's tokens
#pragma unroll
        for (int x = 0; x < CT; ++x) ys[x] = os[x] = zero;
        {
            constexpr int HS = NS * NP * CT > 16 ? NS / 2 : NS;      // slabs requested together: up to 64 registers
#pragma unroll
            for (int s0 = 0; s0 < NS; s0 += HS) {
                DeltaParts<T, NP> f[HS][CT];
#pragma unroll
                for (int sl = 0; sl < HS; ++sl)
#pragma unroll
                    for (int x = 0; x < CT; ++x) f[sl][x] = frag(L::S, s0 + sl, x);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int sl = 0; sl < HS; ++sl)
#pragma unroll
                    for (int x = 0; x < CT; ++x) {
                        DeltaParts<T, 1> k;
                        k.p[0] = K[s0 + sl];
                        ys[x] = delta_mma(k, f[sl][x], ys[x]);
                        if (!BACK) {
                            k.p[0] = Q[s0 + sl];
                            os[x] = delta_mma(k, f[sl][x], os[x]);
                        }
                    }
            }
        }
        load_rows(kb, next, K);
        if (!BACK) load_rows(qb, next, Q);
        if (MODE != DELTA_O)
#pragma unroll
            for (int x = 0; x < CT; ++x)
#pragma unroll
                for (int t = 0; t < TW; ++t) keep(BACK ? a.gm : a.sm, BACK ? 1 : 0, 0, x, u, D, TW * wv + t, S[t][x]);
        if (!BACK) {
#pragma unroll
            for (int x = 0; x < CT; ++x) {
                put(L::Y, wv, x, be * (V[x] - ga4 * ys[x]));
                os[x] = os[x] * (ga4 * a.scale);
            }
            lds_barrier();
            DeltaParts<T, NP> f[CS][CT];
            frags(L::Y, f);
            __builtin_amdgcn_sched_barrier(0);
            f32x4 U[CT];
#pragma unroll
            for (int x = 0; x < CT; ++x) U[x] = zero;
#pragma unroll
            for (int sl = 0; sl < CS; ++sl)
                if (used(sl))
#pragma unroll
                    for (int x = 0; x < CT; ++x) U[x] = delta_mma(A[sl], f[sl][x], U[x]);
            load_tri(ga, next, A);
#pragma unroll
            for (int x = 0; x < CT; ++x) {
                put(L::U, wv, x, U[x] * rh);
                put(L::V, wv, x, U[x]);
            }
            put_most(U);
            lds_barrier();
            DeltaParts<T, NP> f2[CS][CT];
            frags(L::U, f);
            frags(L::V, f2);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < TW; ++t)
#pragma unroll
                for (int x = 0; x < CT; ++x) S[t][x] = S[t][x] * g63;
            load_numbers(next);
            into_state(slice, f);
#pragma unroll
            for (int sl = 0; sl < CS; ++sl)
                if (used(sl))
#pragma unroll
                    for (int x = 0; x < CT; ++x) os[x] = delta_mma(M[sl], f2[sl][x], os[x]);
            load_tri(gm, next, M);
            if (MODE == DELTA_KEEP)
#pragma unroll
                for (int x = 0; x < CT; ++x) keep(a.um, 2, 16, x, u, 64, wv, U[x]);
            put_state();
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = c * CHUNK + P::row(wv, 4 * g + j);
                if (r < len)
#pragma unroll
                    for (int x = 0; x < CT; ++x) *(__attribute__((address_space(1))) T*)(scalar_base(ob + c * vstep, out_at[j]) + 16 * x * ES) = (T)os[x][j];
            }
        } else {
            // dU = diag(rho) K G + M^T dO
#pragma unroll
            for (int x = 0; x < CT; ++x) ys[x] = ys[x] * rh;
#pragma unroll
            for (int sl = 0; sl < CS; ++sl)
                if (used(sl))
#pragma unroll
                    for (int x = 0; x < CT; ++x) {
                        DeltaParts<T, 1> f;
                        f.p[0] = *reinterpret_cast<const Frag*>(smem + L::O + (sl * CT + x) * 1024 + lane * 16);
                        ys[x] = delta_mma(M[sl], f, ys[x]);
                    }
            load_tri(gm, next, M);
#pragma unroll
            for (int x = 0; x < CT; ++x) put(L::Y, wv, x, ys[x]);
            lds_barrier();
            DeltaParts<T, NP> f[CS][CT];
            frags(L::Y, f);
            __builtin_amdgcn_sched_barrier(0);
            f32x4 Y[CT];
#pragma unroll
            for (int x = 0; x < CT; ++x) Y[x] = zero;
#pragma unroll
            for (int sl = 0; sl < CS; ++sl)
                if (used(sl))
#pragma unroll
                    for (int x = 0; x < CT; ++x) Y[x] = delta_mma(A[sl], f[sl][x], Y[x]);
            load_tri(ga, next, A);
            put_most(Y);
#pragma unroll
            for (int x = 0; x < CT; ++x) {
                os[x] = be * Y[x];
                put(L::U, wv, x, -(ga4 * os[x]));
                put(L::V, wv, x, V[x] * (ga4 * a.scale));
            }
            lds_barrier();
            DeltaParts<T, NP> f2[CS][CT];
            frags(L::U, f);
            frags(L::V, f2);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < TW; ++t)
#pragma unroll
                for (int x = 0; x < CT; ++x) S[t][x] = S[t][x] * g63;
            load_numbers(next);
            into_state(slice, f);
            into_state(slice + L::SLICE, f2);
#pragma unroll
            for (int x = 0; x < CT; ++x) keep(a.ym, 3, 16, x, u, 64, wv, Y[x]);
            put_state();
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = c * CHUNK + P::row(wv, 4 * g + j);
                if (r < len)
#pragma unroll
                    for (int x = 0; x < CT; ++x) *(__attribute__((address_space(1))) T*)(scalar_base(ob + c * vstep, out_at[j]) + 16 * x * ES) = (T)os[x][j];
            }
        }
    }
    if (to) {
#pragma unroll
        for (int t = 0; t < TW; ++t)
#pragma unroll
            for (int x = 0; x < CT; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j) to[(size_t)P::row(TW * wv + t, 4 * g + j) * D + col + 16 * x] = S[t][x][j];
    }
}

template <typename T, int D, int NP, int CT, int MODE>
static hipError_t launch(const DeltaArgs& a, hipStream_t stream) {
    typedef ScanLds<T, D, NP, CT, MODE> L;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&delta_scan_kernel<T, D, NP, CT, MODE>), hipFuncAttributeMaxDynamicSharedMemorySize, L::BYTES);
    if (attr != hipSuccess) return attr;
    delta_scan_kernel<T, D, NP, CT, MODE><<<dim3(xcd_deal_grid(D / 16 / CT, a.nseq * a.V)), dim3(256), L::BYTES, stream>>>(a);
    return hipGetLastError();
}
template <typename T, int D, int NP, int MODE>
static hipError_t launch_ct(const DeltaArgs& a, hipStream_t stream) {
    return (long long)a.nseq * a.V * (D / 32) >= 256 ? launch<T, D, NP, 2, MODE>(a, stream) : launch<T, D, NP, 1, MODE>(a, stream);
}
template <int D, int MODE>
static hipError_t launch_np(const DeltaArgs& a, int is_bf16, hipStream_t stream) {
    if (!is_bf16) return launch_ct<float, D, 1, MODE>(a, stream);
    return (MODE == DELTA_BACK ? a.np_b : a.np_f) == 3 ? launch_ct<bf16_t, D, 3, MODE>(a, stream) : launch_ct<bf16_t, D, 2, MODE>(a, stream);
}
hipError_t launch_delta_scan(const DeltaArgs& a, int d, int is_bf16, int mode, hipStream_t stream) {
    if (d == 64) return mode == DELTA_O ? launch_np<64, DELTA_O>(a, is_bf16, stream) : mode == DELTA_KEEP ? launch_np<64, DELTA_KEEP>(a, is_bf16, stream) : launch_np<64, DELTA_BACK>(a, is_bf16, stream);
    return mode == DELTA_O ? launch_np<128, DELTA_O>(a, is_bf16, stream) : mode == DELTA_KEEP ? launch_np<128, DELTA_KEEP>(a, is_bf16, stream) : launch_np<128, DELTA_BACK>(a, is_bf16, stream);
}

}  // namespace path
