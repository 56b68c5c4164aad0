// Attention of a chunk's rows X over a paged cache, bf16.
//
// A workgroup has 128 rows of one key head -- consecutive (token, query head of the group) pairs, 32 per wave -- and a piece of the
// cache, which it walks in stages of 64 cached tokens, brought straight to LDS while the stage before is worked on:
//
//     S^T (32 keys x 32 rows) = K X^T       A = keys (LDS), B = X (registers)
//     O^T (32 d x 32 rows)   += V^T P^T     A = values by transposing reads, B = P (registers, packed from S)
//
// X is computed in fp32 and multiplied as the sum of two bf16 numbers, half as many products again: one alone, or one fp16 number
// against converted keys, leaves every logit of a row off by the same rounding, which the softmax does not average out (log-sum-exp off
// by 2e-6 of itself and more, 1e-7 so).  P is one bf16 number, as everywhere in the library.
// A piece of 16 rows in LDS is 16-byte pieces exchanged as in lds_tile.h, such that neither fragments along a row nor transposing reads
// meet on a bank; the copies fetch them in that order.  Past the end of the sequence and in holes they bring zeros (the buffer's bounds).
// Two workgroups share a CU (64 KB of LDS, 256 registers): the softmax of one runs under the products of the other.  512 rows over 8192 tokens and 2048 over
// 16384, 16 query heads, d = 128: 60 and 405 us (medians under a profiler; 372 at best), 680 TFLOP/s of logits and P V or 1.0 PFLOP/s of products; bound by the matrix units at the clock that
// power leaves them (half of their cycles): without X's second part 82 us less, with a stage's exponentials put between the next one's products, by hand or in a
// pipeline of half stages, the same.  The
// accumulator is rescaled only when a row's maximum has grown by more than 8 (2^8 in P and its sum is exact enough: both are floating).
// Numbered so that the row blocks of a key head and piece run on one XCD, which then reads its keys and values once from memory.
#include <type_traits>

#include "lds_tile.h"
#include "paged_decl.h"

namespace path {

constexpr int PATTN_KEYS = 64;

template <int D> constexpr size_t pattn_smem() { return (size_t)2 * 2 * PATTN_KEYS * D * 2 + 2 * PATTN_KEYS * 4 + 2 * 4 * 4; }

// The four fragments of V^T for a block of 32 d and 64 keys: slab s takes rows 16 s + 4 h + 0..3 and + 8.  The waits are in the block:
// the compiler has a transposing read wait for every copy to LDS.
template <int OFF, int ROWB>
__device__ __forceinline__ void values_tr(unsigned a, unsigned b, bf16x8 (&f)[4]) {
    union U { unsigned long long v[2]; bf16x8 f; } u[4];
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%10\n\tds_read_b64_tr_b16 %1, %9 offset:%10\n\t"
                 "ds_read_b64_tr_b16 %2, %8 offset:%11\n\tds_read_b64_tr_b16 %3, %9 offset:%11\n\t"
                 "ds_read_b64_tr_b16 %4, %8 offset:%12\n\tds_read_b64_tr_b16 %5, %9 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %6, %8 offset:%13\n\tds_read_b64_tr_b16 %7, %9 offset:%13\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(u[0].v[0]), "=&v"(u[0].v[1]), "=&v"(u[1].v[0]), "=&v"(u[1].v[1]), "=&v"(u[2].v[0]), "=&v"(u[2].v[1]), "=&v"(u[3].v[0]), "=&v"(u[3].v[1])
                 : "v"(a), "v"(b), "n"(OFF), "n"(OFF + 16 * ROWB), "n"(OFF + 32 * ROWB), "n"(OFF + 48 * ROWB)
                 : "memory");
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = u[k].f;
}

template <int D, bool GATES>
__global__ __launch_bounds__(256, 2) void paged_attn_kernel(PagedArgs a) {
    typedef TurnedTile<D> L;
    constexpr int ROWB = D * 2, TILE = PATTN_KEYS * ROWB, DS = D / 16, DB = D / 32, PPR = D / 8, RPI = 64 / PPR, GI = 16 / RPI;      // pieces per row, rows and instructions per 16 rows
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];      // [2 stages][keys | values], then (gates) [2 stages][64] c
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, l32 = lane & 31;
    const int Hq = a.H * a.G, blocks = a.row_blocks, units = a.H * a.many_splits;

    // (unit = key head and piece, row block): a unit's blocks on one XCD
    const int slot = blockIdx.x >> 3, unit = __builtin_amdgcn_readfirstlane(slot / blocks) * 8 + (blockIdx.x & 7), block = slot - (slot / blocks) * blocks;
    if (unit >= units) return;
    const int hd = __builtin_amdgcn_readfirstlane(unit % a.H), sp = __builtin_amdgcn_readfirstlane(unit / a.H);
    int s = 0;      // the last sequence whose row blocks start at or before this one
    for (int i = 0; i < a.nseq; i += 64) s += __popcll(__ballot(i + lane < a.nseq && first_block(a, min(i + lane, a.nseq - 1)) <= block));
    s = __builtin_amdgcn_readfirstlane(max(0, s - 1));
    const PagedSeq q = paged_seq(a, s);
    const int n = __builtin_amdgcn_readfirstlane(q.n), m = __builtin_amdgcn_readfirstlane(q.m), t0 = __builtin_amdgcn_readfirstlane(q.t0);
    const int r0 = (block - first_block(a, s)) * 128, pieces = (n + a.many_len - 1) / a.many_len;
    if (m <= a.few_limit || r0 < 0 || r0 >= m * a.G || sp >= pieces) return;
    const int k0 = sp * a.many_len, k1 = min(n, k0 + a.many_len), stages = (k1 - k0 + PATTN_KEYS - 1) / PATTN_KEYS;

    int* const sval = reinterpret_cast<int*>(smem + 4 * TILE + 2 * PATTN_KEYS * 4);      // [2 stages][4] tokens there are in each 16

    // ---- copies: wave w brings the w-th 16 keys and values of a stage ----
    const int* const table = a.table + (long long)s * a.per_seq;
    int ids = -1;
    const int q4 = lane / PPR;      // row within an instruction's
    int voff[GI];
#pragma unroll
    for (int i = 0; i < GI; ++i) {
        const int r = i * RPI + q4;
        voff[i] = r * ROWB + (((lane % PPR) ^ L::turn(r)) << 4);
    }
    auto fetch = [&](int u) {
        if ((u & 63) == 0) {
            const int pos = k0 + (u + lane) * PATTN_KEYS + 16 * wv;
            ids = pos < k1 ? table[pos >> a.page_shift] : -1;
        }
        const int pos = k0 + u * PATTN_KEYS + 16 * wv;
        const PagedGroup p = paged_group(a, __builtin_amdgcn_readlane(ids, u & 63), hd, pos, k1);
        unsigned char* const dst = smem + (u & 1) * 2 * TILE + wv * 16 * ROWB;
        const __amdgpu_buffer_rsrc_t rk = paged_rsrc(a.kpages, p.row, p.valid, ROWB), rv = paged_rsrc(a.vpages, p.row, p.valid, ROWB);
#pragma unroll
        for (int i = 0; i < GI; ++i) {
            paged_to_lds(rk, dst + i * 1024, voff[i]);
            paged_to_lds(rv, dst + TILE + i * 1024, voff[i]);
        }
        if (lane == 0) sval[(u & 1) * 4 + wv] = p.valid;
        if (GATES && lane < 4)
            paged_to_lds(paged_rsrc(a.cpages, p.row, p.valid, 4), smem + 4 * TILE + (u & 1) * PATTN_KEYS * 4 + wv * 64, lane * 16);
    };
    fetch(0);

    // ---- the rows ----
    const int row = r0 + 32 * wv + l32, there = row < m * a.G, tok = (there ? row : m * a.G - 1) / a.G, gq = (there ? row : m * a.G - 1) - tok * a.G;
    const long long at = (long long)(t0 + tok) * Hq + hd * a.G + gq;
    bf16x8 xh[DS], xl[DS];
#pragma unroll
    for (int i = 0; i < DS; ++i) {
        const f32x4* const p = reinterpret_cast<const f32x4*>(a.x + at * D + 16 * i + 8 * h);
        const f32x4 u = p[0], v = p[1];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = e < 4 ? u[e & 3] : v[e & 3];
            xh[i][e] = (bf16_t)x;
            xl[i][e] = (bf16_t)(x - (float)xh[i][e]);
        }
    }
    const float crow = GATES ? a.crow[(long long)(t0 + tok) * a.H + hd] : 0.f, sl2 = a.scale * LOG2E;
    f32x16 O[DB];
#pragma unroll
    for (int b = 0; b < DB; ++b) O[b] = zero16();
    float m_run = -INFINITY, l_run = 0.f;      // (m_run: what the accumulator is scaled to, at most 8 below the maximum)

    const unsigned base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const unsigned kaddr = L::at(l32, 8 * h) * 2;
    const int j16 = l32 & 15;
    const unsigned vaddr = base + L::at(4 * h + (j16 >> 2), (l32 & 16) + 4 * (j16 & 3)) * 2;      // second read: 8 rows on, pieces exchanged by two

    auto stage = [&](int u, auto par) {
        constexpr int PAR = decltype(par)::value, BUF = PAR * 2 * TILE;
        __builtin_amdgcn_s_waitcnt(0x0000);      // this wave's copies have landed; then everybody's, and the other buffer is free
        __syncthreads();
        const int4 valid = *reinterpret_cast<const int4*>(sval + PAR * 4);
        if (u + 1 < stages) fetch(u + 1);
        f32x16 S[2];
        S[0] = S[1] = zero16();
#pragma unroll
        for (int i = 0; i < DS; ++i) {      // two chains of products, neither waiting for its own last one
            const bf16x8 k0 = *reinterpret_cast<const bf16x8*>(smem + BUF + (kaddr ^ (32 * i)));
            const bf16x8 k1 = *reinterpret_cast<const bf16x8*>(smem + BUF + 32 * ROWB + (kaddr ^ (32 * i)));
            S[0] = Tr<bf16_t>::mma(k0, xh[i], S[0]);
            S[1] = Tr<bf16_t>::mma(k1, xh[i], S[1]);
            S[0] = Tr<bf16_t>::mma(k0, xl[i], S[0]);
            S[1] = Tr<bf16_t>::mma(k1, xl[i], S[1]);
        }
        float top = -INFINITY;
        const bool whole = __builtin_amdgcn_readfirstlane(min(min(valid.x, valid.y), min(valid.z, valid.w))) == PAGED_GROUP;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 ck;
                if (GATES) ck = *reinterpret_cast<const f32x4*>(smem + 4 * TILE + PAR * PATTN_KEYS * 4 + (32 * kb + 8 * g + 4 * h) * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (GATES) S[kb][4 * g + e] = S[kb][4 * g + e] * sl2 + (crow - ck[e]) * LOG2E;
                }
            }
        if (!whole)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int v = kb == 0 ? (j < 8 ? valid.x : valid.y) : (j < 8 ? valid.z : valid.w);
                    S[kb][j] = acc_row(j, h) % 16 < v ? S[kb][j] : -INFINITY;
                }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, S[kb][j]);
        {
            const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            top = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1])) * (GATES ? 1.f : sl2);
        }
        if (__any(top > m_run + 8.f)) {
            const float now = fmaxf(m_run, top), f = __builtin_amdgcn_exp2f(m_run - (now == -INFINITY ? 0.f : now));
            m_run = now;
            l_run *= f;
#pragma unroll
            for (int b = 0; b < DB; ++b) O[b] *= f;
        }
        const float ref = m_run == -INFINITY ? 0.f : m_run;
        bf16x8 P[2][2];
        float sum = 0.f;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                S[kb][j] = __builtin_amdgcn_exp2f(GATES ? S[kb][j] - ref : S[kb][j] * sl2 - ref);
                sum += S[kb][j];
            }
            pack_block<bf16_t>(S[kb], P[kb]);
        }
        l_run += sum;
        auto values = [&](auto bt) {
            constexpr int b = decltype(bt)::value;
            const unsigned va = vaddr ^ (64 * b), vb = (va ^ 32) + 8 * ROWB, vc = vaddr ^ (64 * b + 64), vd = (vc ^ 32) + 8 * ROWB;
            bf16x8 v[4], w[4];
            values_tr<BUF + TILE, ROWB>(va, vb, v);
            values_tr<BUF + TILE, ROWB>(vc, vd, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                O[b] = Tr<bf16_t>::mma(v[i], P[i >> 1][i & 1], O[b]);
                O[b + 1] = Tr<bf16_t>::mma(w[i], P[i >> 1][i & 1], O[b + 1]);
            }
        };
        values(std::integral_constant<int, 0>());
        if constexpr (DB == 4) values(std::integral_constant<int, 2>());
    };
    for (int u = 0; u < stages; u += 2) {
        stage(u, std::integral_constant<int, 0>());
        if (u + 1 < stages) stage(u + 1, std::integral_constant<int, 1>());
    }

    // ---- one piece: joined with the new tokens' record and finished; else a record of its own ----
    {
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
        l_run = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    }
    if (!there) return;
    if (pieces == 1) {
        const float m0 = a.many_ml[2 * at], now = fmaxf(m_run, m0), ref = now == -INFINITY ? 0.f : now;
        const float f = __builtin_amdgcn_exp2f(m_run - ref), f0 = __builtin_amdgcn_exp2f(m0 - ref);
        const float l = l_run * f + a.many_ml[2 * at + 1] * f0, inv = 1.f / l;
        const float fi = f * inv, f0i = f0 * inv;
        bf16_t* const o = reinterpret_cast<bf16_t*>(a.o) + at * D;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int d = 32 * b + 8 * g + 4 * h;
                const f32x4 y = *reinterpret_cast<const f32x4*>(a.many_o + at * D + d);
                bf16x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (bf16_t)(O[b][4 * g + e] * fi + y[e] * f0i);
                *reinterpret_cast<bf16x4*>(o + d) = v;
            }
        if (h == 0) a.lse[at] = (now + __builtin_amdgcn_logf(l)) * LN2;
    } else {
        const long long r = at + (long long)(sp + 1) * a.T * Hq;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 v = {O[b][4 * g], O[b][4 * g + 1], O[b][4 * g + 2], O[b][4 * g + 3]};
                *reinterpret_cast<f32x4*>(a.many_o + r * D + 32 * b + 8 * g + 4 * h) = v;
            }
        if (h == 0) { a.many_ml[2 * r] = m_run; a.many_ml[2 * r + 1] = l_run; }
    }
}

template <int D, bool GATES>
static hipError_t launch_pattn_t(const PagedArgs& a, hipStream_t st) {
    constexpr size_t bytes = pattn_smem<D>();
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_attn_kernel<D, GATES>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (attr != hipSuccess) return attr;
    const long long grid = (long long)((a.H * a.many_splits + 7) / 8) * 8 * a.row_blocks;
    if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
    hipLaunchKernelGGL((paged_attn_kernel<D, GATES>), dim3((unsigned)grid), dim3(256), bytes, st, a);
    return hipGetLastError();
}
hipError_t launch_paged_attn(const PagedArgs& a, int d, hipStream_t st) {
    if (a.cpages) return d == 64 ? launch_pattn_t<64, true>(a, st) : launch_pattn_t<128, true>(a, st);
    return d == 64 ? launch_pattn_t<64, false>(a, st) : launch_pattn_t<128, false>(a, st);
}

}  // namespace path
