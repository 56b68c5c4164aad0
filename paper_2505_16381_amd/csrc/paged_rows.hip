// Attention of up to 64 rows over a paged cache, the append of up to 16 new tokens, and both in one pass.
//
// A workgroup has one key head of one sequence and a piece of its cache; its four waves (eight for a short cache) take 32 cached tokens in turn (fp32 and
// some others 16) and meet only at the end.  Everything is 16x16 products, transposed so that activations stay in registers (lane l = 16 g + c):
//
//     S (16 keys x 16 rows)   = K X^T      A = keys as loaded, B = X      result: lane has row c, keys 4 g + i
//     C (16 tokens x 16 keys) = Z K^T      A = Z, B = the same registers  result: lane has key c, tokens 4 g + i
//     K'^T (d x 16 keys)      = K^T - W^T C     result: the key registers, element for element (W^T's rows are numbered so)
//     O^T (d x 16 rows)      += V^T P^T    A = V^T by transposing reads of an LDS tile of the wave's own, B = P
//
// So a key goes from memory to registers and, carried on, from the same registers to memory.  Rows past a sequence's end and holes read
// as zeros and are not written, by the bounds of the buffer that each group of 16 rows is.
// 16-bit operands: keys, values and w are bf16 as stored; X, Z and C are computed in fp32 and multiplied as the sum of two bf16 numbers
// (17 bits: one alone would leave the log-sum-exp of short caches 1e-4 off); P is one bf16 number, as in the library's other kernels.
// Bound by memory: 8 KB of keys and 8 KB of values in flight per wave, up to eight waves per CU.  One token each of 32 sequences of 8192, 16 heads, d = 128, bf16:
// attention 328 us (6.5 TB/s read), with the append 637 (5.1 TB/s, read and written).  Values are read past the caches (hinted; 371 us without), keys are not
// and carried ones are written without a hint (668 with).  Short caches by latency: 500 tokens 15 us, of which the first step takes 9.
// Two steps' keys and values are held at once, 32 tokens each where 256 registers allow it (16 at d = 128 for both operations in one or for 64 rows: spilled
// registers cost 1001 us where it now takes 637).
#include "paged_decl.h"

namespace path {

typedef short v4s __attribute__((ext_vector_type(4)));

template <typename T, int D, int NRT, bool BOTH, int NW> struct RowsCfg {
    static constexpr int ES = sizeof(T), ROWB = D * ES;
    static constexpr int KR = ROWB / 64;                 // 16-byte registers of 16 rows per lane
    static constexpr int U = ES == 2 && !(D == 128 && (NRT == 4 || BOTH)) ? 2 : 1;      // groups of 16 tokens per step: what 256 registers hold two steps of
    static constexpr int PPR = ROWB / 16;                // 16-byte pieces per row
    static constexpr int VBYTES = NW * U * 16 * ROWB;    // value tiles of the waves
    static constexpr int LDX = D + 4;
    // place of piece cp of row r in a value tile: spread over the banks for the reads of 4 (16-bit) or 1 (fp32) row per 16 lanes
    static __device__ __forceinline__ int piece(int r, int cp) {
        if (ES == 2) return r * PPR + (cp ^ (D == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3)));
        return r * PPR + (cp ^ (((r >> 2) & 3) * 4));
    }
    static constexpr size_t floats_before(bool append) { return (size_t)2 * 16 * D + (size_t)16 * NRT * LDX + (append ? 16 * LDX : 0) + 16 * NRT * 17 + 32 + 16 * NRT * 2; }
    static constexpr bool AT_ONCE = NRT == 1;             // LDS has room for all waves' results and another workgroup
    static constexpr size_t PER = NRT * (D / 16) * 1024 + NRT * 512;      // bytes of a wave's
    static constexpr size_t merge_bytes() { return (AT_ONCE ? NW : NW / 2) * PER; }
    static constexpr size_t smem(bool append) {
        const size_t f = (floats_before(append) * 4 + 255) / 256 * 256, a = VBYTES, b = merge_bytes();
        return f + (a > b ? a : b);
    }
};

__device__ __forceinline__ bf16x8 as_bf8(u32x4 v) { union { u32x4 u; bf16x8 f; } x; x.u = v; return x.f; }
__device__ __forceinline__ v4s as_s4(bf16x4 v) { union { bf16x4 f; v4s s; } x; x.f = v; return x.s; }
__device__ __forceinline__ bf16x4 bf4(f32x4 v) { bf16x4 o; for (int i = 0; i < 4; ++i) o[i] = (bf16_t)v[i]; return o; }
__device__ __forceinline__ f32x4 f4(bf16x4 v) { f32x4 o; for (int i = 0; i < 4; ++i) o[i] = (float)v[i]; return o; }
__device__ __forceinline__ f32x4 mma16(v4s a, v4s b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma32(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma4(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// Row c of a matrix in LDS as operand registers: 16-bit: elements 32 s + 8 g + j as a sum of two; fp32: 16 s + 4 g + j.
template <typename T, int D> struct RowOperand;
template <int D> struct RowOperand<bf16_t, D> {
    bf16x8 hi[D / 32], lo[D / 32];
    __device__ __forceinline__ void load(const float* row, int g) {
#pragma unroll
        for (int s = 0; s < D / 32; ++s)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float x = row[32 * s + 8 * g + j];
                hi[s][j] = (bf16_t)x;
                lo[s][j] = (bf16_t)(x - (float)hi[s][j]);
            }
    }
    // keys (as loaded) times this, either way round
    __device__ __forceinline__ f32x4 keys_times(const u32x4* k, f32x4 c) const {
#pragma unroll
        for (int s = 0; s < D / 32; ++s) { c = mma32(as_bf8(k[s]), hi[s], c); c = mma32(as_bf8(k[s]), lo[s], c); }
        return c;
    }
    __device__ __forceinline__ f32x4 times_keys(const u32x4* k, f32x4 c) const {
#pragma unroll
        for (int s = 0; s < D / 32; ++s) { c = mma32(hi[s], as_bf8(k[s]), c); c = mma32(lo[s], as_bf8(k[s]), c); }
        return c;
    }
};
template <int D> struct RowOperand<float, D> {
    f32x4 x[D / 16];
    __device__ __forceinline__ void load(const float* row, int g) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s) x[s] = *reinterpret_cast<const f32x4*>(row + 16 * s + 4 * g);
    }
    __device__ __forceinline__ f32x4 keys_times(const u32x4* k, f32x4 c) const {
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) c = mma4(__uint_as_float(k[s][j]), x[s][j], c);
        return c;
    }
    __device__ __forceinline__ f32x4 times_keys(const u32x4* k, f32x4 c) const {
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) c = mma4(x[s][j], __uint_as_float(k[s][j]), c);
        return c;
    }
};
// -W^T as the left operand of K'^T = K^T - W^T C: lane (row c of a 16-row tile, tokens 4 g + i).  The rows of tile t of the result are
// the elements that a lane of the key registers holds: 16-bit: tile 2 s + u, row r = element 32 s + 8 (r / 4) + 4 u + r % 4; fp32: 16 t + r.
template <typename T, int D> struct Directions;
template <int D> struct Directions<bf16_t, D> {
    v4s w[D / 16];
    __device__ __forceinline__ void load(const float* sw, int c, int g) {
#pragma unroll
        for (int t = 0; t < D / 16; ++t) {
            f32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = -sw[(4 * g + i) * D + 32 * (t >> 1) + 8 * (c >> 2) + 4 * (t & 1) + (c & 3)];
            w[t] = as_s4(bf4(v));
        }
    }
    __device__ __forceinline__ void carry(u32x4* k, f32x4 cc) const {
        const bf16x4 hi = bf4(cc), lo = bf4(cc - f4(hi));
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            const bf16x8 old = as_bf8(k[s]);
            union { bf16x8 f; u32x4 u; } now;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                f32x4 x = {(float)old[4 * u], (float)old[4 * u + 1], (float)old[4 * u + 2], (float)old[4 * u + 3]};
                x = mma16(w[2 * s + u], as_s4(hi), x);
                x = mma16(w[2 * s + u], as_s4(lo), x);
#pragma unroll
                for (int i = 0; i < 4; ++i) now.f[4 * u + i] = (bf16_t)x[i];
            }
            k[s] = now.u;
        }
    }
};
template <int D> struct Directions<float, D> {
    f32x4 w[D / 16];
    __device__ __forceinline__ void load(const float* sw, int c, int g) {
#pragma unroll
        for (int t = 0; t < D / 16; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) w[t][i] = -sw[(4 * g + i) * D + 16 * t + c];
    }
    __device__ __forceinline__ void carry(u32x4* k, f32x4 cc) const {
#pragma unroll
        for (int t = 0; t < D / 16; ++t) {
            union { u32x4 u; f32x4 f; } x;
            x.u = k[t];
#pragma unroll
            for (int i = 0; i < 4; ++i) x.f = mma4(w[t][i], cc[i], x.f);
            k[t] = x.u;
        }
    }
};

// WALK: few new tokens, X and Z formed here; else 16 NRT rows of X from the workspace (no append).
template <typename T, int D, int NRT, bool WALK, bool ATTN, bool APPEND, int NW>
__global__ __launch_bounds__(64 * NW, NW == 4 && NRT == 1 && !(sizeof(T) == 4 && D == 128 && ATTN && APPEND) ? 2 : 1) void paged_rows_kernel(PagedArgs a) {
    using C = RowsCfg<T, D, NRT, ATTN && APPEND, NW>;
    constexpr int NT = 64 * NW;
    constexpr int KR = C::KR, U = C::U, ROWB = C::ROWB, ROWS = 16 * NRT, LDX = C::LDX, DT = D / 16;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    float* const sw = reinterpret_cast<float*>(smem);           // [16][D] w of the new tokens
    float* const skn = sw + 16 * D;                             // [16][D] the new keys
    float* const sx = skn + 16 * D;                             // [ROWS][LDX] X; at the end O
    float* const sz = sx + ROWS * LDX;                          // APPEND: [16][LDX] Z
    float* const sn = sz + (APPEND ? 16 * LDX : 0);             // [ROWS][17] logits with the new tokens
    float* const sb = sn + ROWS * 17;                           // [16] beta, [16] c of the new tokens
    float* const sml = sb + 32;                                 // [ROWS][2] maximum, sum
    unsigned char* const sv = smem + (C::floats_before(APPEND) * 4 + 255) / 256 * 256;      // value tiles; the waves' results

    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
    const int Hq = a.H * a.G;
    int s, h, sp, r0 = 0;
    if constexpr (WALK) {
        const int hs = blockIdx.x % (a.nseq * a.H);
        sp = blockIdx.x / (a.nseq * a.H);
        s = hs / a.H;
        h = hs % a.H;
    } else {
        // (split, tile, head, block of ROWS rows of the tile's 64 G)
        const int per = 64 * a.G / ROWS;
        int x = blockIdx.x;
        const int sub = x % per; x /= per;
        h = x % a.H; x /= a.H;
        const int tile = x % a.tiles;
        sp = x / a.tiles;
        s = 0;      // the last sequence whose tiles start at or before this one
        for (int i = 0; i < a.nseq; i += 64) {
            const bool in = i + lane < a.nseq && first_tile(a, i + lane) <= tile;
            s += __popcll(__ballot(in));
        }
        s = max(0, s - 1);
        r0 = (tile - first_tile(a, s)) * 64 * a.G + sub * ROWS;
    }
    s = __builtin_amdgcn_readfirstlane(s);
    // ---- the pages of this wave's steps, one in each lane (asked for up to the bound: the lengths may still be on their way) ----
    const int* const table = a.table + (long long)s * a.per_seq;
    const int len = WALK ? a.few_len : a.many_len, k0 = sp * len;
    int ids[U];
    auto fetch_ids = [&](int first) {
        const int end = min(a.max_cached, k0 + len);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int pos = k0 + ((first + lane) * NW + wv) * 16 * U + 16 * u;
            ids[u] = pos < end ? table[pos >> a.page_shift] : -1;
        }
    };
    fetch_ids(0);
    const PagedSeq q = paged_seq(a, s);
    const int n = __builtin_amdgcn_readfirstlane(q.n), m = __builtin_amdgcn_readfirstlane(q.m), t0 = __builtin_amdgcn_readfirstlane(q.t0);
    if (WALK ? (m == 0 || m > a.few_limit) : (m <= a.few_limit || r0 >= m * a.G || r0 < 0)) return;
    const int used = WALK ? max(1, (n + len - 1) / len) : (n + len - 1) / len;
    if (sp >= used) return;
    const bool last = WALK && sp == used - 1;
    const int k1 = min(n, k0 + len), rows = min(ROWS, m * a.G - r0);

    struct Step { u32x4 k[U][KR], v[ATTN ? U : 1][ATTN ? KR : 1]; f32x4 cc[U]; long long row[U]; int valid[U]; };
    const int koff = c * ROWB + 16 * g;
    auto fetch = [&](int i, Step& st) {
        if (i > 0 && (i & 63) == 0) fetch_ids(i);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int pos = k0 + (i * NW + wv) * 16 * U + 16 * u;
            const PagedGroup p = paged_group(a, __builtin_amdgcn_readlane(ids[u], i & 63), h, pos, k1);
            st.row[u] = p.row;
            st.valid[u] = p.valid;
            const __amdgpu_buffer_rsrc_t rk = paged_rsrc(a.kpages, p.row, p.valid, ROWB);
#pragma unroll
            for (int r = 0; r < KR; ++r) st.k[u][r] = __builtin_amdgcn_raw_buffer_load_b128(rk, koff + 64 * r, 0, 0);
            if constexpr (ATTN) {
                const __amdgpu_buffer_rsrc_t rv = paged_rsrc(a.vpages, p.row, p.valid, ROWB);
#pragma unroll
                for (int r = 0; r < KR; ++r) st.v[u][r] = __builtin_amdgcn_raw_buffer_load_b128(rv, lane * 16 + 1024 * r, 0, 2);
                if (a.cpages) {
                    union { u32x4 u; f32x4 f; } x;
                    x.u = __builtin_amdgcn_raw_buffer_load_b128(paged_rsrc(a.cpages, p.row, p.valid, 4), 16 * g, 0, 0);
                    st.cc[u] = x.f;
                }
            }
        }
    };
    const int steps = (max(0, k1 - k0 - wv * 16 * U) + 16 * NW * U - 1) / (16 * NW * U);
    Step st0, st1;

    // ---- X (and Z): the new tokens' transitions walked.  Their loads go out before the cache's, so that the walk is not behind those ----
    const T* const wg = reinterpret_cast<const T*>(a.w);
    const T* const kg = reinterpret_cast<const T*>(a.k);
    const T* const vg = reinterpret_cast<const T*>(a.v);
    constexpr int E = D / 16;
    long long new_row = -1;      // APPEND: where token 4 wv + g goes
    if constexpr (WALK) {
        if (APPEND && last && wv < 4 && wv * 4 + g < m) new_row = paged_row(a, s, h, n + wv * 4 + g);
        constexpr int PER_THREAD = (16 * D / 4 + NT - 1) / NT;
        float xw[PER_THREAD][4], xk[PER_THREAD][4], xq[E];
#pragma unroll
        for (int j = 0; j < PER_THREAD; ++j) {
            const int i = j * NT + tid, t = i / (D / 4), e = (i % (D / 4)) * 4;
#pragma unroll
            for (int k = 0; k < 4; ++k) xw[j][k] = xk[j][k] = 0.f;
            if (t < m) {
                load_f32<4>(wg + ((long long)(t0 + t) * a.H + h) * D + e, xw[j]);
                if (last) load_f32<4>(kg + ((long long)(t0 + t) * a.H + h) * D + e, xk[j]);
            }
        }
        const float xb = tid < m ? (float)reinterpret_cast<const T*>(a.beta)[(long long)(t0 + tid) * a.H + h] : 0.f;
        auto query = [&](int r) {
#pragma unroll
            for (int e = 0; e < E; ++e) xq[e] = 0.f;
            if (r < rows) load_f32<E>(reinterpret_cast<const T*>(a.q) + ((long long)(t0 + r / a.G) * Hq + h * a.G + r % a.G) * D + c * E, xq);
        };
        if constexpr (ATTN) query(wv * 4 + g);
        fetch(0, st0);
#pragma unroll
        for (int j = 0; j < PER_THREAD; ++j) {
            const int i = j * NT + tid;
            if (i < 16 * D / 4) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    sw[i * 4 + k] = xw[j][k];
                    if (last) skn[i * 4 + k] = xk[j][k];
                }
            }
        }
        if (tid < 16) sb[tid] = xb;
        if (a.cpages && tid == 64) {
            const long long r = n > 0 ? paged_row(a, s, h, n - 1) : -1;
            float x = r >= 0 ? a.cpages[r] : 0.f;
            for (int t = 0; t < m; ++t) {
                x += (float)reinterpret_cast<const T*>(a.log_f)[(long long)(t0 + t) * a.H + h];
                sb[16 + t] = x;
            }
        }
        __syncthreads();
        if constexpr (ATTN) {
            for (int r = wv * 4 + g; r < ROWS; r += 4 * NW) {
                const int tok = r / a.G;
                float x[E];
                if (r >= 4 * NW) query(r);
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] = xq[e];
                for (int t = m - 1; t >= 0; --t) {
                    if (last) {
                        float y = 0.f;
#pragma unroll
                        for (int e = 0; e < E; ++e) y += x[e] * skn[t * D + c * E + e];
                        y = sum_lanes16(y);
                        if (c == 0) sn[r * 17 + t] = t <= tok ? y : -INFINITY;
                    }
                    float y = 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) y += x[e] * sw[t * D + c * E + e];
                    y = sum_lanes16(y) * (t <= tok ? sb[t] : 0.f);
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] -= y * sw[t * D + c * E + e];
                }
#pragma unroll
                for (int e = 0; e < E; ++e) sx[r * LDX + c * E + e] = x[e];
            }
        }
        if (APPEND && wv < 4) {
            const int t1 = wv * 4 + g;
            float x[E];
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = sw[t1 * D + c * E + e];
            for (int t = m - 2; t >= 0; --t) {
                float y = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) y += x[e] * sw[t * D + c * E + e];
                y = sum_lanes16(y) * (t < t1 ? sb[t] : 0.f);
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] -= y * sw[t * D + c * E + e];
            }
#pragma unroll
            for (int e = 0; e < E; ++e) sz[t1 * LDX + c * E + e] = sb[t1] * x[e];
            if (last && t1 < m) {      // the new token's own row: key carried to the last token, value, gate sum
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] = skn[t1 * D + c * E + e];
                for (int t = 1; t < m; ++t) {
                    float y = 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) y += x[e] * sw[t * D + c * E + e];
                    y = sum_lanes16(y) * (t > t1 ? sb[t] : 0.f);
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] -= y * sw[t * D + c * E + e];
                }
                const long long r = new_row;
                if (r >= 0) {
                    T* const kd = reinterpret_cast<T*>(a.kpages) + r * D + c * E;
                    T* const vd = reinterpret_cast<T*>(a.vpages) + r * D + c * E;
                    const T* const vs = vg + ((long long)(t0 + t1) * a.H + h) * D + c * E;
#pragma unroll
                    for (int e = 0; e < E; ++e) { kd[e] = (T)x[e]; vd[e] = vs[e]; }
                    if (a.cpages && c == 0) a.cpages[r] = sb[16 + t1];
                }
            }
        }
        __syncthreads();
    } else {
        fetch(0, st0);
        for (int i = tid; i < ROWS * D / 4; i += NT) {
            const int r = i / (D / 4), e = (i % (D / 4)) * 4, row = r0 + r;
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
            if (r < rows) x = *reinterpret_cast<const f32x4*>(a.x + ((long long)(t0 + row / a.G) * Hq + h * a.G + row % a.G) * D + e);
            *reinterpret_cast<f32x4*>(sx + r * LDX + e) = x;
        }
        __syncthreads();
    }

    const float sl2 = a.scale * LOG2E;
    RowOperand<T, D> X[ATTN ? NRT : 1], Z;
    Directions<T, D> W;
    float crow[NRT], m_run[NRT], l_run[NRT];
    f32x4 O[ATTN ? NRT : 1][DT];
    if constexpr (ATTN) {
#pragma unroll
        for (int t = 0; t < NRT; ++t) {
            X[t].load(sx + (16 * t + c) * LDX, g);
            const int row = min(16 * t + c, rows - 1);
            crow[t] = !a.cpages ? 0.f : WALK ? sb[16 + row / a.G] : a.crow[(long long)(t0 + (r0 + row) / a.G) * a.H + h];
            m_run[t] = -INFINITY;
            l_run[t] = 0.f;
#pragma unroll
            for (int b = 0; b < DT; ++b) O[t][b] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    if constexpr (APPEND) {
        Z.load(sz + c * LDX, g);
        W.load(sw, c, g);
    }
    unsigned char* const myv = sv + wv * (U * 16 * ROWB);

    auto process = [&](Step& st) {
        f32x4 S[U][NRT];
        if constexpr (ATTN) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int r = 0; r < KR; ++r) {
                    const int p = r * 64 + lane;
                    *reinterpret_cast<u32x4*>(myv + u * 16 * ROWB + C::piece(p / C::PPR, p % C::PPR) * 16) = st.v[u][r];
                }
#pragma unroll
                for (int t = 0; t < NRT; ++t) S[u][t] = X[t].keys_times(st.k[u], f32x4{0.f, 0.f, 0.f, 0.f});
            }
        }
        if constexpr (APPEND) {      // (before the softmax: the stores are on their way, and the keys' registers free)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                W.carry(st.k[u], Z.times_keys(st.k[u], f32x4{0.f, 0.f, 0.f, 0.f}));
                const __amdgpu_buffer_rsrc_t rk = paged_rsrc(a.kpages, st.row[u], st.valid[u], ROWB);
#pragma unroll
                for (int r = 0; r < KR; ++r) __builtin_amdgcn_raw_buffer_store_b128(st.k[u][r], rk, koff + 64 * r, 0, 0);
            }
        }
        if constexpr (ATTN) {
            v4s P16[U][NRT];
#pragma unroll
            for (int t = 0; t < NRT; ++t) {
                float top = -INFINITY;
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float x = S[u][t][i] * sl2;
                        if (a.cpages) x += (crow[t] - st.cc[u][i]) * LOG2E;
                        x = 4 * g + i < st.valid[u] ? x : -INFINITY;
                        S[u][t][i] = x;
                        top = fmaxf(top, x);
                    }
                const float now = fmaxf(m_run[t], max_rows(top)), base = now == -INFINITY ? 0.f : now;
                const float f = __builtin_amdgcn_exp2f(m_run[t] - base);
                m_run[t] = now;
                float sum = 0.f;
#pragma unroll
                for (int u = 0; u < U; ++u) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        S[u][t][i] = __builtin_amdgcn_exp2f(S[u][t][i] - base);
                        sum += S[u][t][i];
                    }
                    if constexpr (sizeof(T) == 2) P16[u][t] = as_s4(bf4(S[u][t]));
                }
                l_run[t] = l_run[t] * f + sum;
#pragma unroll
                for (int b = 0; b < DT; ++b) O[t][b] *= f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const unsigned char* const tile = myv + u * 16 * ROWB;
#pragma unroll
                for (int b = 0; b < DT; ++b) {
                    if constexpr (sizeof(T) == 2) {      // lane j of 16 points at row 4 g + j / 4, columns 16 b + 4 (j % 4) ..; it gets rows 4 g .. + 3 of column 16 b + j
                        const int r = 4 * g + (c >> 2);
                        const v4s vt = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(tile + C::piece(r, 2 * b + ((c & 3) >> 1)) * 16 + 8 * (c & 1)));
#pragma unroll
                        for (int t = 0; t < NRT; ++t) O[t][b] = mma16(vt, P16[u][t], O[t][b]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float vt = *reinterpret_cast<const float*>(tile + C::piece(4 * g + i, 4 * b + (c >> 2)) * 16 + 4 * (c & 3));
#pragma unroll
                            for (int t = 0; t < NRT; ++t) O[t][b] = mma4(vt, S[u][t][i], O[t][b]);
                        }
                    }
                }
            }
        }
    };
    for (int i = 0; i < steps; i += 2) {      // (a step past the end has no valid rows)
        fetch(i + 1, st1);
        process(st0);
        fetch(i + 2, st0);
        process(st1);
    }
    if constexpr (!ATTN) return;

    // ---- the waves' results: the upper half's into the lower's, until one is left ----
    if constexpr (ATTN) {
#pragma unroll
    for (int t = 0; t < NRT; ++t) l_run[t] = sum_rows(l_run[t]);
    constexpr size_t PER = C::PER;
    if constexpr (C::AT_ONCE) {      // all results to LDS; whoever writes an element joins it
        __syncthreads();
        float* const p = reinterpret_cast<float*>(sv + wv * PER);
#pragma unroll
        for (int t = 0; t < NRT; ++t) {
#pragma unroll
            for (int b = 0; b < DT; ++b) *reinterpret_cast<f32x4*>(p + (t * DT + b) * 256 + lane * 4) = O[t][b];
            p[NRT * DT * 256 + t * 128 + lane] = m_run[t];
            p[NRT * DT * 256 + t * 128 + 64 + lane] = l_run[t];
        }
    } else {
    for (int half = NW / 2; half >= 1; half >>= 1) {
        __syncthreads();
        if (wv >= half && wv < 2 * half) {
            float* const p = reinterpret_cast<float*>(sv + (wv - half) * PER);
#pragma unroll
            for (int t = 0; t < NRT; ++t) {
#pragma unroll
                for (int b = 0; b < DT; ++b) *reinterpret_cast<f32x4*>(p + (t * DT + b) * 256 + lane * 4) = O[t][b];
                p[NRT * DT * 256 + t * 128 + lane] = m_run[t];
                p[NRT * DT * 256 + t * 128 + 64 + lane] = l_run[t];
            }
        }
        __syncthreads();
        if (wv < half) {
            const float* const p = reinterpret_cast<const float*>(sv + wv * PER);
#pragma unroll
            for (int t = 0; t < NRT; ++t) {
                const float m2 = p[NRT * DT * 256 + t * 128 + lane], l2 = p[NRT * DT * 256 + t * 128 + 64 + lane];
                const float now = fmaxf(m_run[t], m2), base = now == -INFINITY ? 0.f : now;
                const float f1 = __builtin_amdgcn_exp2f(m_run[t] - base), f2 = __builtin_amdgcn_exp2f(m2 - base);
                m_run[t] = now;
                l_run[t] = l_run[t] * f1 + l2 * f2;
#pragma unroll
                for (int b = 0; b < DT; ++b) O[t][b] = O[t][b] * f1 + *reinterpret_cast<const f32x4*>(p + (t * DT + b) * 256 + lane * 4) * f2;
            }
        }
    }
    if (wv == 0) {
#pragma unroll
        for (int t = 0; t < NRT; ++t) {
#pragma unroll
            for (int b = 0; b < DT; ++b) *reinterpret_cast<f32x4*>(sx + (16 * t + c) * LDX + 16 * b + 4 * g) = O[t][b];
            if (g == 0) { sml[2 * (16 * t + c)] = m_run[t]; sml[2 * (16 * t + c) + 1] = l_run[t]; }
        }
    }
    }
    __syncthreads();

    // ---- the new tokens' keys and values; the result, or this piece's record ----
    for (int i = tid; i < rows * (D / 4); i += NT) {
        const int r = i / (D / 4), e = (i % (D / 4)) * 4, row = r0 + r, tok = row / a.G;
        const long long at = (long long)(t0 + tok) * Hq + h * a.G + row % a.G;
        f32x4 o;
        float mx, l;
        if constexpr (C::AT_ONCE) {
            const int t = r >> 4, from = 16 * ((e & 15) >> 2) + (r & 15);      // the lane that has it
            const float* const p = reinterpret_cast<const float*>(sv);
            constexpr int STEP = PER / 4, ML = NRT * DT * 256;
            float mw[NW];
            mx = -INFINITY;
#pragma unroll
            for (int w = 0; w < NW; ++w) { mw[w] = p[w * STEP + ML + t * 128 + from]; mx = fmaxf(mx, mw[w]); }
            const float ref = mx == -INFINITY ? 0.f : mx;
            o = f32x4{0.f, 0.f, 0.f, 0.f};
            l = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float f = __builtin_amdgcn_exp2f(mw[w] - ref);
                l += f * p[w * STEP + ML + t * 128 + 64 + from];
                o += *reinterpret_cast<const f32x4*>(p + w * STEP + (t * DT + (e >> 4)) * 256 + from * 4) * f;
            }
        } else {
            o = *reinterpret_cast<const f32x4*>(sx + r * LDX + e);
            mx = sml[2 * r];
            l = sml[2 * r + 1];
        }
        if (last) {
            float now = mx;
            auto logit = [&](int t) { return sn[r * 17 + t] * sl2 + (a.cpages ? (sb[16 + tok] - sb[16 + t]) * LOG2E : 0.f); };
            for (int t = 0; t <= tok; ++t) now = fmaxf(now, logit(t));
            const float base = now == -INFINITY ? 0.f : now, f = __builtin_amdgcn_exp2f(mx - base);
            o *= f;
            l *= f;
            mx = now;
            for (int t = 0; t <= tok; ++t) {
                const float p = __builtin_amdgcn_exp2f(logit(t) - base);
                float x[4];
                load_f32<4>(vg + ((long long)(t0 + t) * a.H + h) * D + e, x);
                l += p;
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] += p * x[j];
            }
        }
        if (WALK && used == 1) {
            const float inv = 1.f / l;
            T* const dst = reinterpret_cast<T*>(a.o) + at * D + e;
            typedef T V4 __attribute__((ext_vector_type(4)));
            V4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = (T)(o[j] * inv);
            *reinterpret_cast<V4*>(dst) = v;
            if (e == 0) a.lse[at] = (mx + __builtin_amdgcn_logf(l)) * LN2;
        } else {
            const long long slots = WALK ? (long long)a.nseq * a.few_m * Hq : (long long)a.T * Hq;
            const long long slot = (WALK ? ((long long)s * a.few_m + tok) * Hq + h * a.G + row % a.G : at) + (WALK ? sp : sp + 1) * slots;
            *reinterpret_cast<f32x4*>((WALK ? a.few_o : a.many_o) + slot * D + e) = o;
            if (e == 0) {
                float* const ml = (WALK ? a.few_ml : a.many_ml) + slot * 2;
                ml[0] = mx;
                ml[1] = l;
            }
        }
    }
    }
}

// The records of a row joined, one wave per row; FEW: the pieces of the cache (the last has the new tokens in it), else the new tokens'
// record and the pieces'.
template <typename T, int D, bool FEW>
__device__ __forceinline__ void merge_row(const PagedArgs& a, long long row) {
    const int Hq = a.H * a.G, lane = threadIdx.x & 63;
    int s, tok, used;
    long long at, slot;
    if constexpr (FEW) {
        if (row >= (long long)a.nseq * a.few_m * Hq) return;
        s = (int)(row / ((long long)a.few_m * Hq));
        tok = (int)(row / Hq % a.few_m);
        const PagedSeq q = paged_seq(a, s);
        used = max(1, (q.n + a.few_len - 1) / a.few_len);
        if (tok >= q.m || q.m > a.few_limit || used == 1) return;
        at = (long long)(q.t0 + tok) * Hq + row % Hq;
        slot = row;
    } else {
        if (row >= (long long)a.T * Hq) return;
        tok = (int)(row / Hq);
        s = 0;      // the last sequence that starts at or before the token
        for (int i = 0; i < a.nseq; i += 64) s += __popcll(__ballot(i + lane < a.nseq && a.cu[min(i + lane, a.nseq)] <= tok));
        if (s == 0) return;
        s -= 1;
        const PagedSeq q = paged_seq(a, s);
        if (tok - q.t0 < 0 || tok - q.t0 >= q.m || q.m <= a.few_limit) return;
        used = 1 + (q.n + a.many_len - 1) / a.many_len;
        if (used <= 1 + a.joined) return;      // (the sweep or the attention kernel has finished it)
        at = slot = row;
    }
    constexpr int E = D / 64;
    const long long slots = FEW ? (long long)a.nseq * a.few_m * Hq : (long long)a.T * Hq;
    const float* const po = (FEW ? a.few_o : a.many_o) + slot * D + lane * E;
    const float* const pm = (FEW ? a.few_ml : a.many_ml) + slot * 2;
    float mx = -INFINITY;
    for (int i = 0; i < used; ++i) mx = fmaxf(mx, pm[i * slots * 2]);
    const float base = mx == -INFINITY ? 0.f : mx;
    float l = 0.f, o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    for (int i = 0; i < used; ++i) {
        const float f = __builtin_amdgcn_exp2f(pm[i * slots * 2] - base);
        l += f * pm[i * slots * 2 + 1];
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] += f * po[i * slots * D + e];
    }
    const float inv = 1.f / l;
#pragma unroll
    for (int e = 0; e < E; ++e) reinterpret_cast<T*>(a.o)[at * D + lane * E + e] = (T)(o[e] * inv);
    if (lane == 0) a.lse[at] = (mx + __builtin_amdgcn_logf(l)) * LN2;
}

// Both kinds of sequences in one launch: workgroups of four rows, the first few_blocks for those of few new tokens.
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedArgs a, unsigned few_blocks) {
    const unsigned wv = threadIdx.x >> 6;
    if (blockIdx.x < few_blocks) merge_row<T, D, true>(a, (long long)blockIdx.x * 4 + wv);
    else merge_row<T, D, false>(a, (long long)(blockIdx.x - few_blocks) * 4 + wv);
}

template <typename T, int D, int NRT, bool WALK, bool ATTN, bool APPEND, int NW = 4>
static hipError_t launch_rows_t(const PagedArgs& a, long long grid, hipStream_t st) {
    constexpr size_t bytes = RowsCfg<T, D, NRT, ATTN && APPEND, NW>::smem(APPEND);
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_rows_kernel<T, D, NRT, WALK, ATTN, APPEND, NW>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (attr != hipSuccess) return attr;
    if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
    hipLaunchKernelGGL((paged_rows_kernel<T, D, NRT, WALK, ATTN, APPEND, NW>), dim3((unsigned)grid), dim3(64 * NW), bytes, st, a);
    return hipGetLastError();
}
template <typename T, int D>
static hipError_t launch_rows_d(const PagedArgs& a, hipStream_t st) {
    const long long grid = (long long)a.nseq * a.H * a.few_splits;
    const int rows = a.few_m * a.G;
    if (!a.attn) return launch_rows_t<T, D, 1, true, false, true>(a, grid, st);
    if (rows <= 16 && a.few_waves == 8) return a.append ? launch_rows_t<T, D, 1, true, true, true, 8>(a, grid, st) : launch_rows_t<T, D, 1, true, true, false, 8>(a, grid, st);
    if (a.append) return rows <= 16 ? launch_rows_t<T, D, 1, true, true, true>(a, grid, st) : rows <= 32 ? launch_rows_t<T, D, 2, true, true, true>(a, grid, st) : launch_rows_t<T, D, 4, true, true, true>(a, grid, st);
    return rows <= 16 ? launch_rows_t<T, D, 1, true, true, false>(a, grid, st) : rows <= 32 ? launch_rows_t<T, D, 2, true, true, false>(a, grid, st) : launch_rows_t<T, D, 4, true, true, false>(a, grid, st);
}
hipError_t launch_paged_rows(const PagedArgs& a, int d, int is_bf16, hipStream_t st) {
    if (is_bf16) return d == 64 ? launch_rows_d<bf16_t, 64>(a, st) : launch_rows_d<bf16_t, 128>(a, st);
    return d == 64 ? launch_rows_d<float, 64>(a, st) : launch_rows_d<float, 128>(a, st);
}
template <int D>
static hipError_t launch_rows_many_d(const PagedArgs& a, hipStream_t st) {
    return launch_rows_t<float, D, 4, false, true, false>(a, (long long)a.tiles * a.G * a.H * a.many_splits, st);
}
hipError_t launch_paged_rows_many(const PagedArgs& a, int d, hipStream_t st) { return d == 64 ? launch_rows_many_d<64>(a, st) : launch_rows_many_d<128>(a, st); }
template <typename T, int D>
static hipError_t launch_merge_t(const PagedArgs& a, bool few, bool many, hipStream_t st) {
    const long long fb = few ? ((long long)a.nseq * a.few_m * a.H * a.G + 3) / 4 : 0, mb = many ? ((long long)a.T * a.H * a.G + 3) / 4 : 0;
    hipLaunchKernelGGL((paged_merge_kernel<T, D>), dim3((unsigned)(fb + mb)), dim3(256), 0, st, a, (unsigned)fb);
    return hipGetLastError();
}
hipError_t launch_paged_merge(const PagedArgs& a, bool few, bool many, int d, int is_bf16, hipStream_t st) {
    if (is_bf16) return d == 64 ? launch_merge_t<bf16_t, 64>(a, few, many, st) : launch_merge_t<bf16_t, 128>(a, few, many, st);
    return d == 64 ? launch_merge_t<float, 64>(a, few, many, st) : launch_merge_t<float, 128>(a, few, many, st);
}

}  // namespace path
