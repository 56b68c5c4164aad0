// Gated delta rule: the states, chunk after chunk, and backwards their gradients (delta_decl.h has the formulas).
//
// A wave keeps 16 columns (value indices) of a head's state in registers, all d rows: what it computes needs no other wave.  The chunk's K, Q, A and M come
// through LDS, copied while the chunk before is worked on and shared by the workgroup's NW waves.
#include "delta_parts.h"

namespace path {

enum { DELTA_O = 0, DELTA_KEEP = 1, DELTA_BACK = 2 };      // forward; forward that keeps what the backward needs; backwards

template <typename T, int D, int NP, int NW>
struct ScanLds {
    typedef DeltaOps<T> P;
    static constexpr int TILE = DeltaTile<T, D>::BYTES, TRI = NP * P::NLOW * 1024, ROWS = DELTA_ROWS * 256;
    static constexpr int K = 0, Q = TILE, A = 2 * TILE, M = A + TRI, R = M + TRI, BUF = (R + ROWS + 255) / 256 * 256;
    static constexpr int NB = 2 * BUF <= 160 * 1024 ? 2 : 1, BYTES = NB * BUF;
};

__device__ __forceinline__ void delta_copy16(const void* g, unsigned char* s, unsigned lane_offset) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)scalar_base(g, lane_offset), (__attribute__((address_space(3))) void*)s, 16, 0, 0);
}

// largest |x| of the wave's values as an exponent that leaves fp16 numbers below 2^11
template <int N> __device__ __forceinline__ int delta_exponent(const f32x4* x) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) m = fmaxf(m, fabsf(x[i][j]));
#pragma unroll
    for (int i = 1; i < 64; i *= 2) m = fmaxf(m, __shfl_xor(m, i));
    const int e = (int)(__float_as_uint(m) >> 23) - 127 - 10;
    return e < -126 ? -126 : e;
}

// tile column -> memory, lane n's row of the transposed matrix, as fp32 or as fp16 over 2^ex
template <typename T, int NT> __device__ __forceinline__ void delta_keep(const f32x4* x, void* out, size_t row, int ld, int g, int ex) {
    if constexpr (sizeof(T) == 4) {
        float* const p = static_cast<float*>(out) + row * ld + 4 * g;
#pragma unroll
        for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4*>(p + 16 * t) = x[t];
    } else {
        half_t* const p = static_cast<half_t*>(out) + row * ld + 8 * g;
#pragma unroll
        for (int s = 0; s < NT / 2; ++s) {
            halfx8 h;
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = (half_t)ldexpf(x[2 * s + e / 4][e % 4], -ex);
            *reinterpret_cast<halfx8*>(p + 32 * s) = h;
        }
    }
}

template <typename T, int D, int NP, int NW, int MODE>
__global__ __launch_bounds__(64 * NW, 1) void delta_scan_kernel(DeltaArgs a) {
    typedef DeltaOps<T> P;
    typedef typename P::Frag Frag;
    typedef ScanLds<T, D, NP, NW> L;
    typedef DeltaTile<T, D> Tile;
    constexpr int NS = D / P::SL, NR = D / 16, CS = 64 / P::SL, VEC = 16 / (int)sizeof(T);      // slabs of d, tiles of d, slabs of a chunk
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    int unit, part;
    if (!xcd_deal(blockIdx.x >> 3, blockIdx.x & 7, NR / NW, a.nseq * a.V, unit, part)) return;
    const int s = __builtin_amdgcn_readfirstlane(unit / a.V), hv = unit - s * a.V, hk = __builtin_amdgcn_readfirstlane(hv / a.G);
    const DeltaSeq sq = delta_seq(a, s);
    const int len = __builtin_amdgcn_readfirstlane(sq.len), tile0 = __builtin_amdgcn_readfirstlane(sq.tile0);
    if (a.slots && len <= a.few) return;
    const int NC = (len + CHUNK - 1) / CHUNK;
    const int col = 16 * (part * NW + wv) + n;      // the lane's value index

    // the first state: of a pool's slot, given, or zeros.  Rows of tile t: delta_row(t, 4 g + j)
    f32x4 S[NR];
    const size_t head = ((size_t)s * a.V + hv) * D * D;
    const float* from = nullptr;
    float* to = nullptr;
    if (MODE == DELTA_BACK) {
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
    for (int t = 0; t < NR; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) S[t][j] = from ? from[(size_t)P::row(t, 4 * g + j) * D + col] : 0.f;

    const T* const kp = static_cast<const T*>(a.k) + delta_at(a, sq, s, a.ks, a.kt) + hk * a.kh;
    const T* const qp = static_cast<const T*>(a.q) + delta_at(a, sq, s, a.ks, a.kt) + hk * a.kh;
    const long long vat = delta_at(a, sq, s, a.vs, a.vt) + hv * a.vh + col;
    const T* const vp = static_cast<const T*>(MODE == DELTA_BACK ? a.d_o : a.v) + vat;
    T* const op = static_cast<T*>(MODE == DELTA_BACK ? a.dv : a.o) + vat;
    const char *const ga = static_cast<const char*>(MODE == DELTA_BACK ? a.at : a.a), *const gm = static_cast<const char*>(MODE == DELTA_BACK ? a.mt : a.m);

    // Copies of a chunk to LDS, 1 KB each, dealt to the waves.  Rows behind the sequence's end are its last one again: their beta is 0.
    auto copies = [&](int c, unsigned char* buf) {
        const size_t u = (size_t)(tile0 + c) * a.V + hv;
        const int last = len - 1 - c * CHUNK;
        constexpr int RPI = 1024 / Tile::ROWB;      // rows of an instruction
        const int r = lane / Tile::PPR, x = lane % Tile::PPR;
        for (int i = wv; i < 64 / RPI; i += NW) {
            const int row = i * RPI + r, held = row < last ? row : last;
            const unsigned off = (unsigned)((x ^ Tile::turn(row)) * 16);
            const T* const k0 = kp + (long long)(c * CHUNK + held) * a.kt;
            const T* const q0 = qp + (long long)(c * CHUNK + held) * a.kt;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(reinterpret_cast<const char*>(k0) + off),
                                             (__attribute__((address_space(3))) void*)(buf + L::K + i * 1024), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(reinterpret_cast<const char*>(q0) + off),
                                             (__attribute__((address_space(3))) void*)(buf + L::Q + i * 1024), 16, 0, 0);
        }
        for (int i = wv; i < L::TRI / 1024; i += NW) {
            delta_copy16(ga + u * L::TRI + i * 1024, buf + L::A + i * 1024, lane * 16);
            delta_copy16(gm + u * L::TRI + i * 1024, buf + L::M + i * 1024, lane * 16);
        }
        const char* const rows = reinterpret_cast<const char*>(a.rows + u * DELTA_ROWS * 64);
        if (wv == 0) delta_copy16(rows, buf + L::R, lane * 16);
        if (wv == NW - 1 && lane < 16) delta_copy16(rows + 1024, buf + L::R + 1024, lane * 16);
    };
    auto values = [&](int c, T (&v)[4][4]) {      // the lane's column of V (backwards: dO)
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = c * CHUNK + P::row(t, 4 * g + j), held = r < len ? r : len - 1;
                v[t][j] = vp[held * a.vt];
            }
    };

    const int step = MODE == DELTA_BACK ? -1 : 1, first = MODE == DELTA_BACK ? NC - 1 : 0;
    T vn[4][4];
    if (NC > 0) {
        copies(first, smem);
        values(first, vn);
    }
    unsigned char* buf = smem;
    for (int i = 0; i < NC; ++i) {
        const int c = first + i * step;
        __builtin_amdgcn_s_waitcnt(0x0000);      // this wave's copies have landed; then everybody's, and the other buffer is free
        __syncthreads();
        f32x4 V[4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) V[t][j] = c * CHUNK + P::row(t, 4 * g + j) < len ? (float)vn[t][j] : 0.f;
        if (i + 1 < NC) {
            if (L::NB == 2) copies(c + step, buf == smem ? smem + L::BUF : smem);
            values(c + step, vn);
        }
        const float* const rows = reinterpret_cast<const float*>(buf + L::R);
        auto of_row = [&](int which, int t) { return *reinterpret_cast<const f32x4*>(rows + which * 64 + P::row(t, 4 * g)); };      // of the lane's four tokens of tile t
        const unsigned nat = Tile::nat(n, g);
        auto along = [&](int tile, int t, int sl) { DeltaParts<T, 1> f; f.p[0] = *reinterpret_cast<const Frag*>(buf + tile + ((nat ^ (64 * sl)) + Tile::tile_off(t))); return f; };
        auto tri = [&](int mat, int at) {
            DeltaParts<T, NP> f;
#pragma unroll
            for (int p = 0; p < NP; ++p) f.p[p] = reinterpret_cast<const Frag*>(buf + mat)[(p * P::NLOW + at) * 64 + lane];
            return f;
        };
        // tiles of the state += (tile in LDS)^T x, x in slabs of the chunk
        auto into_state = [&](int tile, const DeltaParts<T, NP>* x) {
            if constexpr (sizeof(T) == 2) {
                const unsigned base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)(buf + tile);
#pragma unroll
                for (int tp = 0; tp < NR / 2; ++tp) {
                    bf16x8 f[2][2];
                    delta_ld_tr<D>(base + (delta_tr<D>(lane) ^ (64 * tp)), f);
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int sl = 0; sl < 2; ++sl) {
                            DeltaParts<T, 1> y;
                            y.p[0] = f[b][sl];
                            S[2 * tp + b] = delta_mma(y, x[sl], S[2 * tp + b]);
                        }
                }
            } else {
#pragma unroll
                for (int t = 0; t < NR; ++t)
#pragma unroll
                    for (int sl = 0; sl < CS; ++sl) {
                        DeltaParts<T, 1> y;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int row = 16 * sl + 4 * g + e, cc = 16 * t + n;
                            y.p[0][e] = *reinterpret_cast<const float*>(buf + tile + row * Tile::ROWB + (((cc >> 2) ^ Tile::turn(row)) << 4) + (cc & 3) * 4);
                        }
                        S[t] = delta_mma(y, x[sl], S[t]);
                    }
            }
        };
        const size_t u = (size_t)(tile0 + c) * a.V + hv;
        const float g63 = rows[64 + 63];

        if (MODE == DELTA_KEEP || MODE == DELTA_BACK) {
            int ex = 0;
            if constexpr (sizeof(T) == 2) {
                ex = delta_exponent<NR>(S);
                if (lane == 0) a.ex[u * 32 + (MODE == DELTA_BACK ? 8 : 0) + part * NW + wv] = ex;
            }
            delta_keep<T, NR>(S, MODE == DELTA_BACK ? a.gm : a.sm, u * D + col, D, g, ex);
        }
        DeltaParts<T, NP> Sp[NS];
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) delta_pack<T, NP>(S, sl, Sp[sl]);
        f32x4 x[4];      // K S
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            x[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int sl = 0; sl < NS; ++sl) x[t] = delta_mma(along(L::K, t, sl), Sp[sl], x[t]);
        }
        if (MODE != DELTA_BACK) {
            f32x4 o[4];      // scale diag(gamma) Q S
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int sl = 0; sl < NS; ++sl) o[t] = delta_mma(along(L::Q, t, sl), Sp[sl], o[t]);
                const f32x4 be = of_row(0, t), ga4 = of_row(1, t);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[t][j] = be[j] * (V[t][j] - ga4[j] * x[t][j]);
                    o[t][j] *= a.scale * ga4[j];
                }
            }
            DeltaParts<T, NP> y[CS];
#pragma unroll
            for (int sl = 0; sl < CS; ++sl) delta_pack<T, NP>(x, sl, y[sl]);
            f32x4 U[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                U[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int sl = 0; sl < CS; ++sl)
                    if (P::low(t, sl)) U[t] = delta_mma(tri(L::A, P::low_at(t, sl)), y[sl], U[t]);
            }
            if (MODE == DELTA_KEEP) {
                int ex = 0;
                if constexpr (sizeof(T) == 2) {
                    ex = delta_exponent<4>(U);
                    if (lane == 0) a.ex[u * 32 + 16 + part * NW + wv] = ex;
                }
                delta_keep<T, 4>(U, a.um, u * D + col, 64, g, ex);
            }
#pragma unroll
            for (int sl = 0; sl < CS; ++sl) delta_pack<T, NP>(U, sl, y[sl]);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int sl = 0; sl < CS; ++sl)
                    if (P::low(t, sl)) o[t] = delta_mma(tri(L::M, P::low_at(t, sl)), y[sl], o[t]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = c * CHUNK + P::row(t, 4 * g + j);
                    if (r < len) op[r * a.vt] = (T)o[t][j];
                }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) U[t] = U[t] * of_row(2, t);
#pragma unroll
            for (int sl = 0; sl < CS; ++sl) delta_pack<T, NP>(U, sl, y[sl]);
#pragma unroll
            for (int t = 0; t < NR; ++t) S[t] = S[t] * g63;
            into_state(L::K, y);
        } else {
            DeltaParts<T, 1> dO[CS];
#pragma unroll
            for (int sl = 0; sl < CS; ++sl) delta_pack<T, 1>(V, sl, dO[sl]);
#pragma unroll
            for (int t = 0; t < 4; ++t) {      // dU = diag(rho) K G + M^T dO
                x[t] = x[t] * of_row(2, t);
#pragma unroll
                for (int sl = 0; sl < CS; ++sl)
                    if (P::up(t, sl)) x[t] = delta_mma(tri(L::M, P::up_at(t, sl)), dO[sl], x[t]);
            }
            DeltaParts<T, NP> y[CS];
#pragma unroll
            for (int sl = 0; sl < CS; ++sl) delta_pack<T, NP>(x, sl, y[sl]);
            f32x4 Y[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                Y[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int sl = 0; sl < CS; ++sl)
                    if (P::up(t, sl)) Y[t] = delta_mma(tri(L::A, P::up_at(t, sl)), y[sl], Y[t]);
            }
            int ex = 0;
            if constexpr (sizeof(T) == 2) {
                ex = delta_exponent<4>(Y);
                if (lane == 0) a.ex[u * 32 + 24 + part * NW + wv] = ex;
            }
            delta_keep<T, 4>(Y, a.ym, u * D + col, 64, g, ex);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const f32x4 be = of_row(0, t), ga4 = of_row(1, t);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = c * CHUNK + P::row(t, 4 * g + j);
                    const float z = be[j] * Y[t][j];
                    if (r < len) op[r * a.vt] = (T)z;
                    Y[t][j] = -ga4[j] * z;
                    V[t][j] *= a.scale * ga4[j];
                }
            }
#pragma unroll
            for (int t = 0; t < NR; ++t) S[t] = S[t] * g63;
#pragma unroll
            for (int sl = 0; sl < CS; ++sl) delta_pack<T, NP>(Y, sl, y[sl]);
            into_state(L::K, y);
#pragma unroll
            for (int sl = 0; sl < CS; ++sl) delta_pack<T, NP>(V, sl, y[sl]);
            into_state(L::Q, y);
        }
        if (L::NB == 2) {
            buf = buf == smem ? smem + L::BUF : smem;
        } else if (i + 1 < NC) {
            __syncthreads();
            copies(c + step, buf);
        }
    }
    if (to) {
#pragma unroll
        for (int t = 0; t < NR; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) to[(size_t)P::row(t, 4 * g + j) * D + col] = S[t][j];
    }
}

template <typename T, int D, int NP, int NW, int MODE>
static hipError_t launch(const DeltaArgs& a, hipStream_t stream) {
    typedef ScanLds<T, D, NP, NW> L;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&delta_scan_kernel<T, D, NP, NW, MODE>), hipFuncAttributeMaxDynamicSharedMemorySize, L::BYTES);
    if (attr != hipSuccess) return attr;
    delta_scan_kernel<T, D, NP, NW, MODE><<<dim3(xcd_deal_grid(D / 16 / NW, a.nseq * a.V)), dim3(64 * NW), L::BYTES, stream>>>(a);
    return hipGetLastError();
}
template <typename T, int D, int NP, int MODE>
static hipError_t launch_nw(const DeltaArgs& a, hipStream_t stream) {
    const long long blocks = (long long)a.nseq * a.V * (D / 16);
    if (D == 128 && sizeof(T) == 2 && blocks >= 8 * 256) return launch<T, D, NP, sizeof(T) == 2 ? D / 16 : 4, MODE>(a, stream);
    if (blocks >= 4 * 256) return launch<T, D, NP, 4, MODE>(a, stream);
    return launch<T, D, NP, 2, MODE>(a, stream);
}
template <int D, int MODE>
static hipError_t launch_np(const DeltaArgs& a, int is_bf16, hipStream_t stream) {
    if (!is_bf16) return launch_nw<float, D, 1, MODE>(a, stream);
    return (MODE == DELTA_BACK ? a.np_b : a.np_f) == 3 ? launch_nw<bf16_t, D, 3, MODE>(a, stream) : launch_nw<bf16_t, D, 2, MODE>(a, stream);
}
hipError_t launch_delta_scan(const DeltaArgs& a, int d, int is_bf16, int mode, hipStream_t stream) {
    if (d == 64) return mode == DELTA_O ? launch_np<64, DELTA_O>(a, is_bf16, stream) : mode == DELTA_KEEP ? launch_np<64, DELTA_KEEP>(a, is_bf16, stream) : launch_np<64, DELTA_BACK>(a, is_bf16, stream);
    return mode == DELTA_O ? launch_np<128, DELTA_O>(a, is_bf16, stream) : mode == DELTA_KEEP ? launch_np<128, DELTA_KEEP>(a, is_bf16, stream) : launch_np<128, DELTA_BACK>(a, is_bf16, stream);
}

}  // namespace path
