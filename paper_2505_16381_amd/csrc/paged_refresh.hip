// The cached keys of a paged cache carried on by a chunk of new tokens: k <- k + (H_{m-1} .. H_0 - I) k, in place.
//
// The d x d matrix comes from the scan over the chunk's tiles (paged_chunk16.hip, fp32 paged_chunk.hip).  As products of 16 keys at a time, K'^T = K^T + M K^T
// with M's rows numbered so that a lane's results are the elements that it loaded: from memory to registers to memory.  16-bit: a wave
// holds all of M (128 registers at d = 128) and takes every fourth group of 16 keys.  M's elements are at most 2, transitions being contractions, and one fp16 number
// each; a key is brought to [1, 2) by a power of two before it is made fp16 numbers and back after the product, so that keys of any size are carried alike
// (as they stood, those from 65520 on became infinite and those below 2^-25 were not carried).  fp32: M lies in LDS.
// Bound by memory: every key read and written once, three groups of a wave on their way (16 heads of 8192, d = 128: 18 us, 3.7 TB/s, of which scaling takes 1; with one group on its way 6 more).
#include "paged_decl.h"

namespace path {

template <typename T, int D> constexpr size_t refresh_smem() { return sizeof(T) == 4 ? (size_t)D * (D + 4) * 4 : 0; }

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void paged_refresh_kernel(PagedArgs a) {
    constexpr int ROWB = D * (int)sizeof(T), KR = ROWB / 64;
    extern __shared__ __attribute__((aligned(16))) float sm[];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
    const int hs = blockIdx.x % (a.nseq * a.H), s = hs / a.H, h = hs % a.H, k0 = blockIdx.x / (a.nseq * a.H) * a.refresh_len;
    const PagedSeq q = paged_seq(a, s);
    const int n = __builtin_amdgcn_readfirstlane(q.n);
    if (q.m <= a.few_limit || k0 >= n) return;
    const int k1 = min(n, k0 + a.refresh_len);
    const int* const table = a.table + (long long)s * a.per_seq;
    const int mine = k0 + (lane * 4 + wv) * 16, id = mine < k1 ? table[mine >> a.page_shift] : -1;
    const int koff = c * ROWB + 16 * g;
    u32x4 k[KR], kn[KR], k2[KR], k3[KR];
    auto fetch = [&](int i, u32x4* k) {
        const int pos = k0 + (i * 4 + wv) * 16;
        const PagedGroup p = paged_group(a, i < 64 ? __builtin_amdgcn_readlane(id, i & 63) : -1, h, pos, k1);
        const __amdgpu_buffer_rsrc_t r = paged_rsrc(a.kpages, p.row, p.valid, ROWB);
#pragma unroll
        for (int j = 0; j < KR; ++j) k[j] = __builtin_amdgcn_raw_buffer_load_b128(r, koff + 64 * j, 0, 0);
        return p;
    };
    PagedGroup p = fetch(0, k);
    if constexpr (sizeof(T) == 2) {
        PagedGroup p1 = fetch(1, kn), p2 = fetch(2, k2);
        const half_t* const M = reinterpret_cast<const half_t*>(a.pt) + (size_t)hs * D * D;
        halfx8 f[D / 16][D / 32];
#pragma unroll
        for (int t = 0; t < D / 16; ++t)
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
                f[t][j] = *reinterpret_cast<const halfx8*>(M + (32 * (t >> 1) + 8 * (c >> 2) + 4 * (t & 1) + (c & 3)) * D + 32 * j + 8 * g);
        auto carry = [&](const PagedGroup& p, const u32x4* k) {
            halfx8 kh[KR];
            union { u32x4 u; bf16x8 b; } x[KR];
            // the key's exponent: that of its largest element, in the four lanes that have it (as an integer, which orders bf16 numbers without their sign)
            unsigned even = 0, odd = 0;
#pragma unroll
            for (int j = 0; j < KR; ++j) {
                x[j].u = k[j];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    even = max(even, k[j][e] << 16 & 0x7f800000u);
                    odd = max(odd, k[j][e] & 0x7f800000u);
                }
            }
            const unsigned top = __float_as_uint(max_rows(__uint_as_float(max(even, odd))));
            const unsigned expo = min(max(top, 1u << 23), 253u << 23);
            const float down = __uint_as_float((254u << 23) - expo), up = __uint_as_float(expo);      // 2^(127 - e), 2^(e - 127)
#pragma unroll
            for (int j = 0; j < KR; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) kh[j][e] = (half_t)((float)x[j].b[e] * down);
            __builtin_amdgcn_sched_barrier(0);      // (products between the conversions would need more registers than there are)
#pragma unroll
            for (int t = 0; t < D / 16; ++t) {
                f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < D / 32; ++j) y = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[t][j], kh[j], y, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[t >> 1].b[4 * (t & 1) + e] = (bf16_t)((float)x[t >> 1].b[4 * (t & 1) + e] + y[e] * up);
            }
            const __amdgpu_buffer_rsrc_t r = paged_rsrc(a.kpages, p.row, p.valid, ROWB);
#pragma unroll
            for (int j = 0; j < KR; ++j) __builtin_amdgcn_raw_buffer_store_b128(x[j].u, r, koff + 64 * j, 0, 0);
        };
        // three groups on their way (past the end: none)
        for (int i = 0; k0 + (i * 4 + wv) * 16 < k1; i += 4) {
            const PagedGroup p3 = fetch(i + 3, k3);
            carry(p, k);
            p = fetch(i + 4, k);
            carry(p1, kn);
            p1 = fetch(i + 5, kn);
            carry(p2, k2);
            p2 = fetch(i + 6, k2);
            carry(p3, k3);
        }
    } else {
        constexpr int LD = D + 4;
        const float* const M = reinterpret_cast<const float*>(a.pt) + (size_t)hs * D * D;
        for (int i = tid; i < D * D / 4; i += 256) {
            const int r = i / (D / 4), e = (i % (D / 4)) * 4;
            *reinterpret_cast<f32x4*>(sm + r * LD + e) = *reinterpret_cast<const f32x4*>(M + r * D + e);
        }
        __syncthreads();
        for (int i = 0; k0 + (i * 4 + wv) * 16 < k1; ++i) {
            const PagedGroup pn = fetch(i + 1, kn);
            const __amdgpu_buffer_rsrc_t r = paged_rsrc(a.kpages, p.row, p.valid, ROWB);
#pragma unroll
            for (int t = 0; t < D / 16; ++t) {
                union { u32x4 u; f32x4 f; } y;
                y.u = k[t];
#pragma unroll
                for (int j = 0; j < KR; ++j) {
                    const f32x4 f = *reinterpret_cast<const f32x4*>(sm + (16 * t + c) * LD + 16 * j + 4 * g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) y.f = __builtin_amdgcn_mfma_f32_16x16x4f32(f[e], __uint_as_float(k[j][e]), y.f, 0, 0, 0);
                }
                __builtin_amdgcn_raw_buffer_store_b128(y.u, r, koff + 64 * t, 0, 0);
            }
            p = pn;
#pragma unroll
            for (int j = 0; j < KR; ++j) k[j] = kn[j];
        }
    }
}

template <typename T, int D>
static hipError_t launch_refresh_t(const PagedArgs& a, hipStream_t st) {
    constexpr size_t bytes = refresh_smem<T, D>();
    static const hipError_t attr = bytes ? hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_refresh_kernel<T, D>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) : hipSuccess;
    if (attr != hipSuccess) return attr;
    const long long grid = (long long)a.nseq * a.H * ((a.max_cached + a.refresh_len - 1) / a.refresh_len);
    if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
    hipLaunchKernelGGL((paged_refresh_kernel<T, D>), dim3((unsigned)grid), dim3(256), bytes, st, a);
    return hipGetLastError();
}
hipError_t launch_paged_refresh(const PagedArgs& a, int d, int is_bf16, hipStream_t st) {
    if (is_bf16) return d == 64 ? launch_refresh_t<bf16_t, 64>(a, st) : launch_refresh_t<bf16_t, 128>(a, st);
    return d == 64 ? launch_refresh_t<float, 64>(a, st) : launch_refresh_t<float, 128>(a, st);
}

}  // namespace path
