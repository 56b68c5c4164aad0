// Paged caches: argument struct, device-side views and launchers of the kernels that attend to them and append to them.
//
// A sequence's n cached keys are carried to its last token, khat_i = H_{n-1} .. H_{i+1} k_i (H_t = I - beta_t w_t w_t^T).
// Of m new tokens, A = strictLower(W W^T), T = (I + diag(beta) A)^{-1} diag(beta), Z = T W, D = strictLower(W K^T),
// L = lower(Q W^T) (diagonal included):
//
//     H_{m-1} .. H_0 = I - W^T Z                          what the append applies to every cached key
//     X = Q - (L T) W          rows H_0 .. H_a q_a        what the cached keys are multiplied with
//     Q K^T - L (T D)          for b <= a                 logits among the new tokens
//     K - (T D)^T W            rows H_{m-1} .. H_{b+1} k_b   the new keys as they are cached
//
// A sequence goes one of two ways, by its own number of new tokens (few_limit).  Few: every workgroup forms X and Z itself by
// walking the tokens' transitions (paged_rows.hip), and one pass over the cache does the attention, the append or both.  More:
// tiles of 64 new tokens (paged_chunk16.hip, fp32 paged_chunk.hip) leave X, the attention among the new tokens and H_{m-1} .. H_0;
// then the cache is attended to (paged_attn.hip, fp32 paged_rows.hip) and carried on (paged_refresh.hip).
#pragma once
#include "path_common.h"

namespace path {

constexpr int PAGED_FEW = 16;         // most new tokens, and PAGED_FEW_ROWS most rows (token, query head of the group), of the one-pass way
constexpr int PAGED_FEW_ROWS = 64;
constexpr int PAGED_GROUP = 16;       // cached tokens that share a lookup of their page: every page is a multiple of it

struct PagedArgs {
    const void *q, *k, *v, *w, *beta, *log_f;      // [T][H*G][d], [T][H][d], [T][H]
    void *kpages, *vpages;                         // [num_pages][H][page][d]
    float* cpages;                                 // [num_pages][H][page], NULL without gates
    const int *table, *cached, *cu;                // [nseq][per_seq], [nseq], [nseq + 1]
    void* o;                                       // [T][H*G][d]
    float* lse;                                    // [T][H*G]
    int nseq, T, max_new, max_cached, num_pages, page_shift, per_seq, H, G;
    float scale;
    int attn, append;
    // sequences of at most few_limit new tokens: the cache in few_splits pieces of few_len tokens; records of the pieces
    int few_limit, few_m, few_splits, few_len, few_waves;
    float *few_o, *few_ml;                         // [split][nseq * few_m * H * G][d], [..][2]
    // the others: tiles of 64 new tokens (tile c of sequence s: first_tile(s) + c < tiles)
    int tiles, many_splits, many_len;
    int refresh_len;                               // cached tokens per workgroup that carries them on, at most 4096
    int row_blocks;                                // blocks of 128 rows, first_block(s) + i < row_blocks
    int joined;                                    // the attention kernel joins a single piece with record 0 itself
    float *x, *crow;                               // [T][H*G][d] X; [T][H] c of the new tokens (gates)
    float *many_o, *many_ml;                       // [1 + split][T * H * G][d], [..][2]; record 0: the new tokens' own
    void *kt, *wt, *zt, *vt;                       // [tiles][H]: operand tiles of the new tokens, see paged_chunk.hip (bf16: kt, zt only, [hi, lo][tiles][H])
    float* sd;                                     // [tiles][H*G][64][64] logits inside a tile
    void* pt;                                      // [nseq][H][d][d]: H_{m-1} .. H_0 - I of all new tokens (fp32; with bf16 fp16)
};

struct PagedSeq { int n, t0, m; };
// Lengths as they stand in device memory, held to the bounds that the call was given.
__device__ __forceinline__ PagedSeq paged_seq(const PagedArgs& a, int s) {
    const int n = min(max(a.cached[s], 0), a.max_cached);
    const int t0 = min(max(a.cu[s], 0), a.T), t1 = min(max(a.cu[s + 1], t0), a.T);
    return {n, t0, min(t1 - t0, a.max_new)};
}
// The tiles of a sequence start here: sequences before it have at most t0 / 64 + s tiles, each at most one part tile.
__device__ __forceinline__ int first_tile(const PagedArgs& a, int s) { return (min(max(a.cu[s], 0), a.T) >> 6) + s; }
// The same for blocks of 128 rows (token, query head of the group).
__device__ __forceinline__ int first_block(const PagedArgs& a, int s) { return min(max(a.cu[s], 0), a.T) * a.G / 128 + s; }

// Where 16 cached tokens of a head lie, and how many of them there are: pos a multiple of 16 below n.  An entry of the page table outside the
// pool is a hole: nothing is read or written there.
struct PagedGroup { long long row; int valid; };
__device__ __forceinline__ PagedGroup paged_group(const PagedArgs& a, int page, int h, int pos, int n) {
    const bool hole = (unsigned)page >= (unsigned)a.num_pages;
    const long long row = (((long long)(hole ? 0 : page) * a.H + h) << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
    return {row, hole ? 0 : max(0, min(PAGED_GROUP, n - pos))};
}
// The place of token pos (cached or about to be) of sequence s; -1 in a hole or past the table.
__device__ __forceinline__ long long paged_row(const PagedArgs& a, int s, int h, int pos) {
    const int i = pos >> a.page_shift;
    if (i >= a.per_seq) return -1;
    const int page = a.table[(long long)s * a.per_seq + i];
    if ((unsigned)page >= (unsigned)a.num_pages) return -1;
    return (((long long)page * a.H + h) << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
}

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
// Rows of a group as a buffer: accesses past the valid ones read zeros and write nothing.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t paged_rsrc(const void* pages, long long row, int valid, int row_bytes) {
    const unsigned long long p = reinterpret_cast<unsigned long long>(pages) + (unsigned long long)row * row_bytes;
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)p), hi = __builtin_amdgcn_readfirstlane((unsigned)(p >> 32));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((unsigned long long)hi << 32 | lo), 0,
                                             __builtin_amdgcn_readfirstlane(valid * row_bytes), 0x00020000);
}

// 16 bytes per lane of such a buffer straight to LDS, one lane behind the other.  (Written inside a kernel template, the builtin keeps the host pass from
// emitting the kernel: a function
// of its own.)
__device__ __forceinline__ void paged_to_lds(__amdgpu_buffer_rsrc_t r, unsigned char* lds, int offset) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)lds, 16, offset, 0, 0, 0);
}

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.693147180559945309417f;

// value over the four 16-lane rows of a wave
__device__ __forceinline__ float max_rows(float v) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
    const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ float sum_rows(float v) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(y[0]) + __uint_as_float(y[1]);
}
// sum over the 16 lanes of a row, in every one of them
__device__ __forceinline__ float sum_lanes16(float x) {
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x128, 0xf, 0xf, true));
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x124, 0xf, 0xf, true));
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x122, 0xf, 0xf, true));
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x121, 0xf, 0xf, true));
    return x;
}
// Whether one of N registers of four is an infinity or NaN (by the bits: comparisons take NaN for absent)
template <int N> __device__ __forceinline__ bool not_finite(const f32x4* x) {
    unsigned top = 0;
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(x[t][i]) & 0x7fffffffu);
    return top >= 0x7f800000u;
}
// E consecutive elements as fp32
template <int E, typename T> __device__ __forceinline__ void load_f32(const T* p, float* x) {
    typedef T V __attribute__((ext_vector_type(E)));
    const V v = *reinterpret_cast<const V*>(p);
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = (float)v[e];
}

hipError_t launch_paged_rows(const PagedArgs& a, int d, int is_bf16, hipStream_t st);       // few new tokens: everything; d = 64, 128
hipError_t launch_paged_rows_many(const PagedArgs& a, int d, hipStream_t st);               // X rows from the workspace, fp32
hipError_t launch_paged_attn(const PagedArgs& a, int d, hipStream_t st);                    // the same, bf16
hipError_t launch_paged_merge(const PagedArgs& a, bool few, bool many, int d, int is_bf16, hipStream_t st);      // records joined, of either way or both
hipError_t launch_paged_chunk(const PagedArgs& a, int d, hipStream_t st);                   // tiles of the new tokens, fp32
hipError_t launch_paged_sweep(const PagedArgs& a, int d, hipStream_t st);                   // attention among the new tokens, X
hipError_t launch_paged_scan(const PagedArgs& a, int d, hipStream_t st);                    // the new keys, H_{m-1} .. H_0
hipError_t launch_paged_chunk16(const PagedArgs& a, int d, hipStream_t st);                 // bf16: the tiles
hipError_t launch_paged_sweep16(const PagedArgs& a, int d, hipStream_t st);                 // sweep and scan in one launch
hipError_t launch_paged_refresh(const PagedArgs& a, int d, int is_bf16, hipStream_t st);    // cached keys <- H_{m-1} .. H_0 keys

}  // namespace path
