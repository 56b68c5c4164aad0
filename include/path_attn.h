/*
 * path_attn.h -- C ABI of the PaTH attention hot path for AMD MI355X (gfx950).
 *
 * PaTH attention (paper Sec. 2.2) is causal softmax attention whose logit is
 *
 *     s_ij = scale * q_i^T H_i H_{i-1} ... H_{j+1} k_j ,   H_t = I - beta_t w_t w_t^T ,
 *
 * (j <= i; empty product for j = i), with o_i = sum_j softmax_j(s_ij) v_j and
 * lse_i = log sum_j exp(s_ij).  The library evaluates it with the paper's
 * blockwise algorithm (Sec. 3.2-3.3): per chunk of 64 tokens a UT transform
 * (triangular solve) gives boundary-adjusted queries/keys and the chunk's
 * transition product; a FlashAttention-style right-to-left sweep over key
 * chunks then applies that product to the resident query tile after each
 * chunk.  All arithmetic runs in hand-written gfx950 kernels.
 *
 * Conventions common to every entry point
 *  - Every data pointer is DEVICE memory owned by the caller.  The library
 *    never allocates, frees or synchronises; all kernels are enqueued on
 *    `stream` (a hipStream_t passed as void*, NULL = the null stream).
 *  - Layout: q, k, v, w, o, d_o, dq, dk, dv, dw are contiguous [B, H, L, d];
 *    beta, dbeta, lse are contiguous [B, H, L] (the *_layout and *_varlen entry
 *    points also take [B, L, H, d] and packed sequences).  w and beta are per
 *    token and per head.  No grouped-query sharing (but for the path_paged_* calls).
 *  - dtype `dt` is the storage type of q,k,v,w,beta,o and of all gradients
 *    (PATH_F32: float, PATH_BF16: bfloat16).  lse is always float.
 *  - Arithmetic.  PATH_F32 contracts on fp32 MFMA throughout.  PATH_BF16 accumulates
 *    in fp32 and contracts on 16-bit MFMA with TWO operand types: the softmax
 *    probabilities, the values and d_o are bf16 operands; everything the method
 *    TRANSPORTS -- the query state, the boundary-adjusted keys, the chunk products
 *    I - P, the matrices inside the chunk transform, and in the backward the
 *    gradients of the query state and of the chunk products -- are fp16 operands
 *    (11-bit significand: bf16's 8 bits there put the log-sum-exp 1e-3 .. 3e-3
 *    off; same MFMA rate).
 *  - Range rule for PATH_BF16 (a consequence of the fp16 operands; fp16 ends at
 *    65504, no status code reports a violation): the transitions are contractions
 *    for beta in [0,2], |w| <= 1, so every transported quantity is bounded by the
 *    Euclidean norms of the rows of q and k -- those norms must stay below 65504;
 *    in the backward the state gradients are bounded by
 *    scale * L * max|d_o| * max|v| * max_row|k| and must stay below it too.  Beyond
 *    the bound (or for beta, w outside those ranges, where products can grow with
 *    L) results are UNDEFINED: infinities or NaNs may appear in any output, never
 *    a fault.  Magnitudes below 6e-8 (fp16's smallest subnormal) flush to zero in
 *    the transported operands.  PATH_F32 has fp32's range throughout.
 *  - d must be 64 or 128; any L >= 1 (a ragged last chunk is handled inside).
 *  - `scale` multiplies the finished bilinear form (the paper's logits are
 *    unscaled: pass 1.0f for those); it must be > 0 (else PATH_ERR_UNSUPPORTED).
 *    lse uses the natural logarithm.
 *  - w is used as given (no normalisation), beta as given (no clipping).
 *  - Only causal attention is defined by the method (the transition product
 *    runs along the path j -> i): causal == 0 returns PATH_ERR_UNSUPPORTED.
 *  - `workspace` is caller-owned device scratch of at least
 *    path_attn_workspace_bytes(...) bytes, 256-byte aligned; its contents are
 *    undefined afterwards.  Calls that share a workspace must be ordered on
 *    one stream.
 *  - Errors are reported by return code before anything is launched (bad
 *    arguments) or after a failed launch (PATH_ERR_HIP); the library never
 *    aborts or throws.  Outputs are fully overwritten on PATH_OK.
 *  - Threads: entry points may be called from several host threads at once as
 *    long as the calls use different workspaces (and streams as the caller sees
 *    fit).  The first launch of each kernel instantiation in a process sets a
 *    launch attribute once; that is guarded (std::call_once), so concurrent first
 *    calls are safe.  path_attn_last_error is per thread.
 *  - Determinism: every result except PaTH-FoX's dlog_f is bit-reproducible run
 *    to run (no atomics, fixed summation order).  dlog_f sums its column and row
 *    sums in shared memory in no fixed order: reproducible up to fp32 rounding of
 *    those sums.
 */
#ifndef PATH_ATTN_H
#define PATH_ATTN_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { PATH_F32 = 0, PATH_BF16 = 1 } path_dtype_t;

/* Layout of the caller's tensors, for the entry points that take one (the others use PATH_LAYOUT_BHLD):
 *   PATH_LAYOUT_BHLD: q, k, v, w, o and gradients [B,H,L,d]; beta, lse, log_f and gradients [B,H,L]
 *   PATH_LAYOUT_BLHD: ...                          [B,L,H,d]; ...                             [B,L,H]
 * (both contiguous, d innermost). */
typedef enum { PATH_LAYOUT_BHLD = 0, PATH_LAYOUT_BLHD = 1 } path_layout_t;

typedef enum {
    PATH_OK = 0,
    PATH_ERR_NULL = 1,        /* a required pointer is NULL                         */
    PATH_ERR_SHAPE = 2,       /* B,H,L < 1, d not in {64,128}, or sizes overflow     */
    PATH_ERR_DTYPE = 3,       /* dt is not PATH_F32 / PATH_BF16                      */
    PATH_ERR_UNSUPPORTED = 4, /* causal == 0, or scale <= 0                          */
    PATH_ERR_WORKSPACE = 5,   /* workspace too small or misaligned                   */
    PATH_ERR_HIP = 6,         /* a kernel launch failed                              */
    PATH_ERR_ALIGN = 7        /* q,k,v,w,o (or a gradient) not 16-byte aligned       */
} path_status_t;

/* Human-readable name of a status code (static storage, never NULL). */
const char* path_status_str(path_status_t status);

/* After an entry point returned PATH_ERR_HIP on this thread: which step failed
 * and the runtime's name for the error, e.g. "forward sweep: hipErrorInvalidValue (1)".
 * The entry points clear, on entry, a runtime error state left behind by other code in
 * the process and note it here ("inherited and cleared on entry: ...") without failing.
 * Thread-local storage owned by the library, never NULL; empty before any such event. */
const char* path_attn_last_error(void);

/* Bytes of device workspace needed by path_attn_fwd (for_backward == 0) or
 * path_attn_bwd (for_backward != 0) for this problem.  Returns 0 for
 * arguments the entry points would reject. */
size_t path_attn_workspace_bytes(int B, int H, int L, int d, path_dtype_t dt, int for_backward);

/* A memory-bounded backward.  path_attn_bwd (and path_attn_fox_bwd, path_attn_bwd_layout, path_attn_varlen_bwd)
 * accept ANY workspace that holds at least one head: every (batch, head) is an independent problem, so with less
 * than path_attn_workspace_bytes(..., 1) the backward passes over the heads in groups of as many as fit -- the
 * same kernels on smaller grids, the same arithmetic, bit-identical gradients; the price is more launches and,
 * for small groups, a GPU that is not filled.  The query states that dominate the workspace (one per (query
 * chunk, key block) pair) are stored only for the group in flight.
 *   path_attn_bwd_workspace_bytes_for_heads: bytes that let `heads` (clamped to B*H) heads pass together;
 *     heads = 1 is the minimum any backward accepts.  0 for arguments the entry points reject.
 *   path_attn_bwd_heads_per_pass: heads per pass a workspace of that size gives (0: too small even for one).
 * The training pair (path_attn_train_*) keeps the states of ALL heads between its two calls and needs the full size. */
size_t path_attn_bwd_workspace_bytes_for_heads(int B, int H, int L, int d, path_dtype_t dt, int heads);
int path_attn_bwd_heads_per_pass(int B, int H, int L, int d, path_dtype_t dt, size_t workspace_bytes);

/* Introspection for tests and profiling: byte offsets, inside the forward
 * workspace, of the five intermediates the chunk-preprocessing kernel (paper
 * Sec. 3.2) hands to the sweep kernel, in this order: boundary-adjusted key
 * tiles, V^T tiles, negated chunk-product tiles (I - P), boundary-adjusted
 * queries (fp32), diagonal-block logits (fp32); offsets[5] = end of the last of them
 * (further regions follow, up to path_attn_workspace_bytes).
 * Returns PATH_ERR_SHAPE / PATH_ERR_DTYPE for arguments the forward rejects. */
path_status_t path_attn_fwd_workspace_layout(int B, int H, int L, int d, path_dtype_t dt,
                                             size_t offsets[6]);

/*
 * Forward (paper Sec. 2.2 definition; Sec. 3.2-3.3 blockwise algorithm).
 *   in : q, k, v, w [B,H,L,d] (dt), beta [B,H,L] (dt)       -- device, read-only
 *   out: o [B,H,L,d] (dt), lse [B,H,L] (float)              -- device
 */
path_status_t path_attn_fwd(const void* q, const void* k, const void* v, const void* w,
                            const void* beta, void* o, float* lse,
                            int B, int H, int L, int d, int causal, float scale,
                            path_dtype_t dt, void* workspace, size_t workspace_bytes,
                            void* stream);

/*
 * The two stages of the forward as separate launches, for callers that want
 * to time or overlap them; path_attn_fwd is exactly path_attn_fwd_prep
 * followed by path_attn_fwd_sweep on the same stream and workspace.
 *   prep  (Sec. 3.2): chunk UT transform -> workspace (reads q,k,v,w,beta)
 *   sweep (Sec. 3.3): right-to-left scan over key chunks -> o, lse (reads workspace only)
 * Same argument rules and error codes as path_attn_fwd.
 */
path_status_t path_attn_fwd_prep(const void* q, const void* k, const void* v, const void* w,
                                 const void* beta, int B, int H, int L, int d, path_dtype_t dt,
                                 void* workspace, size_t workspace_bytes, void* stream);
path_status_t path_attn_fwd_sweep(void* o, float* lse, int B, int H, int L, int d, float scale,
                                  path_dtype_t dt, void* workspace, size_t workspace_bytes,
                                  void* stream);

/*
 * Backward of loss = sum(d_o * o) (the paper states no backward; this is the
 * reverse-mode derivative of the forward above, through the chunk transform).
 *   in : q, k, v, w, beta as in the forward; o, lse as the forward wrote them;
 *        d_o [B,H,L,d] (dt)                                  -- device, read-only
 *   out: dq, dk, dv, dw [B,H,L,d] (dt), dbeta [B,H,L] (dt)   -- device
 * dw is the gradient with respect to the w passed in (no projection onto the
 * unit sphere).  Results are bit-reproducible: every sum is taken in a fixed order.
 */
path_status_t path_attn_bwd(const void* q, const void* k, const void* v, const void* w,
                            const void* beta, const void* o, const float* lse, const void* d_o,
                            void* dq, void* dk, void* dv, void* dw, void* dbeta,
                            int B, int H, int L, int d, int causal, float scale,
                            path_dtype_t dt, void* workspace, size_t workspace_bytes,
                            void* stream);

/*
 * PaTH-FoX (paper Sec. 2.2, "Extension: PaTH-FoX"): the attention weight of key j for query i
 * gets the extra factor prod_{s=j+1..i} f_s of data-dependent forget gates f_s in (0,1), i.e.
 * the logit becomes  scale * q_i^T H_i ... H_{j+1} k_j + sum_{s=j+1..i} log f_s.
 * log_f [B,H,L] (dt, device, read-only) holds the LOG of the gates (<= 0); everything else as
 * in path_attn_fwd, same workspace size.  lse is the log-sum-exp of the full logits.
 */
path_status_t path_attn_fox_fwd(const void* q, const void* k, const void* v, const void* w,
                                const void* beta, const void* log_f, void* o, float* lse,
                                int B, int H, int L, int d, int causal, float scale,
                                path_dtype_t dt, void* workspace, size_t workspace_bytes,
                                void* stream);

/* Backward of path_attn_fox_fwd: as path_attn_bwd, plus dlog_f [B,H,L] (dt), the gradient with
 * respect to log_f (entry 0 of every head is exactly 0: the first gate lies on no path).
 * Same workspace size as path_attn_bwd. */
path_status_t path_attn_fox_bwd(const void* q, const void* k, const void* v, const void* w,
                                const void* beta, const void* log_f, const void* o, const float* lse,
                                const void* d_o, void* dq, void* dk, void* dv, void* dw, void* dbeta,
                                void* dlog_f, int B, int H, int L, int d, int causal, float scale,
                                path_dtype_t dt, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Training pair: forward and backward of one step that share a workspace, so that the chunk
 * transform (paper Sec. 3.2) and the recurrence of the query states (Sec. 3.3) run once per step
 * instead of once in each: the forward's sweep also writes the states the backward starts from.
 * path_attn_train_fwd
 * computes o and lse exactly as path_attn_fwd (log_f == NULL) or path_attn_fox_fwd (log_f given)
 * do, but in a workspace of the BACKWARD's size (path_attn_workspace_bytes(..., for_backward = 1)),
 * where it leaves the transformed operands and the query states; path_attn_train_bwd then computes the gradients exactly
 * as path_attn_bwd / path_attn_fox_bwd do (dlog_f given iff log_f is), provided that the workspace
 * has not been written since path_attn_train_fwd returned and that q, k, v, w, beta, log_f are the
 * same tensors with the same contents.  The price is that the workspace stays alive between the
 * two calls.  Arguments, layouts and error codes as for the calls they stand in for.
 */
path_status_t path_attn_train_fwd(const void* q, const void* k, const void* v, const void* w,
                                  const void* beta, const void* log_f, void* o, float* lse,
                                  int B, int H, int L, int d, int causal, float scale,
                                  path_dtype_t dt, void* workspace, size_t workspace_bytes, void* stream);
/* path_attn_train_fwd as two launches, for callers that time or overlap the stages: it is exactly
 * path_attn_train_fwd_prep followed by path_attn_train_fwd_sweep on the same stream and workspace
 * (with_gates != 0 iff log_f was given to the first). */
path_status_t path_attn_train_fwd_prep(const void* q, const void* k, const void* v, const void* w,
                                       const void* beta, const void* log_f, int B, int H, int L, int d,
                                       path_dtype_t dt, void* workspace, size_t workspace_bytes, void* stream);
path_status_t path_attn_train_fwd_sweep(void* o, float* lse, int with_gates, int B, int H, int L, int d, float scale,
                                        path_dtype_t dt, void* workspace, size_t workspace_bytes, void* stream);
path_status_t path_attn_train_bwd(const void* q, const void* k, const void* v, const void* w,
                                  const void* beta, const void* log_f, const void* o, const float* lse,
                                  const void* d_o, void* dq, void* dk, void* dv, void* dw, void* dbeta,
                                  void* dlog_f, int B, int H, int L, int d, int causal, float scale,
                                  path_dtype_t dt, void* workspace, size_t workspace_bytes, void* stream);

/* path_attn_train_bwd in stages, for callers that time them (bench.py brackets each with events): `stages` is a
 * set of PATH_BWD_STAGE_* bits; the selected stages are enqueued in the order of their values.  Calling it with
 * one stage after the other, in that order, is exactly path_attn_train_bwd (which is `stages` = PATH_BWD_STAGE_ALL);
 * a later stage reads what the earlier ones left in the workspace.  Unknown or no bits: PATH_ERR_UNSUPPORTED. */
enum {
    PATH_BWD_STAGE_SCAN = 1,       /* dO tiles and delta; adjoint scan over the key blocks (dQ-side)          */
    PATH_BWD_STAGE_KEYS_NEAR = 2,  /* PATH_F32: key-side sums inside a super-block (PATH_BF16: in _CHUNK)     */
    PATH_BWD_STAGE_KEYS_FAR = 4,   /* key-side sums over all queries right of the key's super-block          */
    PATH_BWD_STAGE_DDP = 8,        /* PATH_F32: gradients of the products (PATH_BF16: the key-side passes)   */
    PATH_BWD_STAGE_CHUNK = 16,     /* adjoint of the second level and of the chunk transform: the gradients;
                                    * PATH_BF16: first the key-side sums inside the key's own super-block    */
    PATH_BWD_STAGE_ALL = 31
};
path_status_t path_attn_train_bwd_stages(int stages, const void* q, const void* k, const void* v, const void* w,
                                         const void* beta, const void* log_f, const void* o, const float* lse,
                                         const void* d_o, void* dq, void* dk, void* dv, void* dw, void* dbeta,
                                         void* dlog_f, int B, int H, int L, int d, int causal, float scale,
                                         path_dtype_t dt, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The forward and backward on either layout.  log_f == NULL: plain PaTH (as path_attn_fwd / path_attn_bwd);
 * log_f given: PaTH-FoX (as path_attn_fox_fwd / path_attn_fox_bwd; dlog_f is required iff log_f is).
 * Same workspace sizes, argument rules and error codes; an unknown layout returns PATH_ERR_UNSUPPORTED.
 * The kernels read and write the caller's tensors in place through their strides: nothing is transposed
 * or copied.
 */
path_status_t path_attn_fwd_layout(const void* q, const void* k, const void* v, const void* w,
                                   const void* beta, const void* log_f, void* o, float* lse,
                                   int B, int H, int L, int d, path_layout_t layout, int causal, float scale,
                                   path_dtype_t dt, void* workspace, size_t workspace_bytes, void* stream);
path_status_t path_attn_bwd_layout(const void* q, const void* k, const void* v, const void* w,
                                   const void* beta, const void* log_f, const void* o, const float* lse,
                                   const void* d_o, void* dq, void* dk, void* dv, void* dw, void* dbeta,
                                   void* dlog_f, int B, int H, int L, int d, path_layout_t layout, int causal,
                                   float scale, path_dtype_t dt, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Variable-length batches: nseq sequences packed along the token axis, q, k, v, w, o and gradients
 * [T,H,d], beta, lse, log_f and gradients [T,H] (T = cu_seqlens[nseq]); sequence s owns the tokens
 * cu_seqlens[s] .. cu_seqlens[s+1]-1 and attends only to itself.  cu_seqlens is a HOST array of nseq+1
 * ints (cu_seqlens[0] = 0, strictly increasing; else PATH_ERR_SHAPE); it is read before the call returns
 * (copied to the head of the workspace on `stream`).
 * The whole batch is ONE set of kernel launches: sequence s is batch entry s of a problem whose workspace
 * arrays are sized for the longest sequence, every kernel takes its bounds from the entry's own length, and
 * workgroups beyond a shorter sequence's end exit at once -- results are bit-identical to calling the
 * fixed-length entry points sequence by sequence on [1,L_s,H,d] tensors.  The workspace must hold
 * path_attn_varlen_workspace_bytes(...) bytes: the sequence table plus path_attn_workspace_bytes(nseq, H,
 * longest length, ...); the backward also accepts less, down to the table plus one head's worth (see the
 * memory-bounded backward above).  log_f / dlog_f as above.
 */
size_t path_attn_varlen_workspace_bytes(const int* cu_seqlens, int nseq, int H, int d, path_dtype_t dt,
                                        int for_backward);
path_status_t path_attn_varlen_fwd(const void* q, const void* k, const void* v, const void* w,
                                   const void* beta, const void* log_f, void* o, float* lse,
                                   const int* cu_seqlens, int nseq, int H, int d, int causal, float scale,
                                   path_dtype_t dt, void* workspace, size_t workspace_bytes, void* stream);
path_status_t path_attn_varlen_bwd(const void* q, const void* k, const void* v, const void* w,
                                   const void* beta, const void* log_f, const void* o, const float* lse,
                                   const void* d_o, void* dq, void* dk, void* dv, void* dw, void* dbeta,
                                   void* dlog_f, const int* cu_seqlens, int nseq, int H, int d, int causal,
                                   float scale, path_dtype_t dt, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Decode path (paper Sec. 3.4 "Efficient Inference").  Caches are caller-owned device memory,
 * kcache and vcache [B,H,Lmax,d] contiguous in the I/O type dt; position i of a head holds
 * token i.  The key cache holds REFRESHED keys: after t tokens, k_i^(t) = H_t ... H_{i+1} k_i
 * (the section's first equation applied at every arrival), so that attention of q_t over the
 * cache is ordinary softmax attention.  With dt = PATH_BF16 every refresh rounds the stored
 * keys to bf16 again; that rounding is part of the method as the paper runs it.
 *
 * path_key_prefill: fills positions [0, L) of both caches after a prompt of L tokens (the
 * section's key-prefill formula, with suffix products: linear in L).  It reads the forward
 * workspace of the SAME prompt, i.e. call it after path_attn_fwd / path_attn_fwd_prep on
 * (q, k, v, w, beta) with that workspace (device, read-only here); v [B,H,L,d] is copied.  (The workspace of a
 * training pair will not do: nothing to the right of a prompt is ever asked of a training step, which leaves the last
 * 1024 tokens' keys where the chunk transform put them.)
 * Errors: PATH_ERR_SHAPE also for L > Lmax.
 *
 * path_decode_step: one arriving token per (batch, head): q, k, v, w [B,H,d], beta [B,H] (dt,
 * device, read-only).  n = tokens already cached (0 <= n < Lmax).  Refreshes the n cached
 * keys in place, appends k and v at position n, writes o [B,H,d] (dt) and lse [B,H] (fp32,
 * natural log) of the attention of q over the n+1 keys.  workspace: device scratch of
 * path_decode_workspace_bytes(B, H, d) bytes, 256-byte aligned, contents undefined afterwards.
 * Nothing is allocated; all work is enqueued on `stream`.
 */
size_t path_decode_workspace_bytes(int B, int H, int d);
path_status_t path_key_prefill(const void* v, int B, int H, int L, int d, path_dtype_t dt,
                               const void* fwd_workspace, size_t fwd_workspace_bytes,
                               void* kcache, void* vcache, int Lmax, void* stream);
path_status_t path_decode_step(const void* q, const void* k, const void* v, const void* w,
                               const void* beta, void* kcache, void* vcache, int n, int Lmax,
                               void* o, float* lse, int B, int H, int d, float scale,
                               path_dtype_t dt, void* workspace, size_t workspace_bytes,
                               void* stream);

/*
 * PaTH-FoX at decode time (paper Sec. 2.2 "Extension: PaTH-FoX" applied to the decoding step of Sec. 3.4): key i's
 * logit gets sum_{s=i+1..t} log f_s.  The running sums c_i = sum_{s<=i} log f_s of the cached tokens are a third
 * cache, `ccache` [B,H,Lmax] fp32 (natural logarithm, caller-owned device memory like the other two).
 *   path_gate_prefill     fills ccache[.., 0..L) from the prompt's gates log_f [B,H,L] (I/O type).
 *   path_decode_step_fox  path_decode_step with the arriving token's log gate log_f [B,H] (I/O type): uses
 *                         c_n = c_{n-1} + log f_n (c_{-1} = 0), adds c_n - c_i to key i's logit (nothing to the
 *                         token's own) and appends c_n to ccache.  Everything else -- caches, workspace, errors --
 *                         as for path_decode_step.
 */
path_status_t path_gate_prefill(const void* log_f, int B, int H, int L, path_dtype_t dt, float* ccache, int Lmax,
                                void* stream);
path_status_t path_decode_step_fox(const void* q, const void* k, const void* v, const void* w, const void* beta,
                                   const void* log_f, void* kcache, void* vcache, float* ccache, int n, int Lmax,
                                   void* o, float* lse, int B, int H, int d, float scale, path_dtype_t dt,
                                   void* workspace, size_t workspace_bytes, void* stream);

/*
 * Serving from paged caches (Sec. 3.4 with sequences of different lengths, several new tokens a call, and cache memory handed out
 * in pages).  The caches hold what the decode path's hold -- keys carried to the sequence's last token, k_i^(n) = H_{n-1} .. H_{i+1} k_i,
 * and values; with gates the running sums c_i -- in pools of pages:
 *   kpages, vpages [num_pages, H, page_size, d] (dt), cpages [num_pages, H, page_size] (fp32; NULL for plain PaTH).
 *   page_size a power of two from 16 to 4096; slot j of a head in page p holds the tokens i with page_table[s][i / page_size] = p, i % page_size = j.
 * Lengths and tables are DEVICE int32 arrays, read when the kernels run (a captured call follows them through its replays):
 *   page_table [nseq, pages_per_seq]; cached [nseq], tokens of each sequence in the cache; cu_new [nseq + 1], not decreasing: sequence s
 *   brings the new tokens cu_new[s] .. cu_new[s+1]-1 of q, k, v, w, beta, log_f, o, lse, packed along the token axis.  No new tokens, none cached: allowed.
 * Host arguments bound them: T tokens in the packed tensors, at most max_new new and max_cached cached tokens a sequence (both choose the
 * grids and how the cache is split; close bounds are fast).  Values past the bounds are held to them; rows of o and lse that belong to no sequence are left
 * as they are.  A page_table entry outside [0, num_pages) is a hole: its tokens take no part, nothing is read or written
 * there (a gate sum that would have been read there counts as 0).
 *
 * Shapes: q, o [T, H * group, d], lse [T, H * group] (fp32); k, v, w [T, H, d]; beta, log_f [T, H]; all contiguous.  Query heads
 * h * group .. h * group + group - 1 share key head h with its w, beta and gates (group 1: as everywhere else).
 *
 *   path_paged_attn    o, lse of the new tokens: each attends to its sequence's cached tokens and to the new ones up to itself.  The
 *                      caches are only read (drafted tokens can be looked at and dropped; pages may be shared between sequences).
 *   path_paged_append  the new tokens' transitions applied to the cached keys, in place, and the new keys (carried to the last new token),
 *                      values and gate sums written behind them.  The caller owns `cached` and adds the new tokens to it
 *                      afterwards.  Room: tokens past pages_per_seq * page_size are not stored.  Pages that it reaches belong to one sequence only
 *                      (keys carried on by two sequences are nobody's: copy the pages first; the call then leaves undefined keys, no fault).
 *   path_paged_extend  both, in the order attention, append; up to 16 new tokens and 64 rows (new tokens x group) a sequence in one pass over its cache.
 *
 * Attention uses the cached keys as they stand: the logit is formed from x = H_{n} .. H_{n+a} q with the stored key, where path_decode_step
 * rounds the refreshed key first.  A server may put appends off: the new tokens of path_paged_attn are then all tokens since the
 * last append (keys are read and written back, and rounded, once per append instead of once per token).
 * Arithmetic with PATH_BF16: what is computed from the inputs -- X, the carried keys, the transitions -- is multiplied as the sum of two bf16 numbers, with
 * bf16's range (log-sum-exp 5e-7 off in the mean, single rows up to 6e-6), probabilities as one.  The one exception: the product of a chunk's transitions that its append applies to
 * the cached keys is an fp16 operand, beta and w being held to the range rule above; the keys there are scaled by powers of two and may have any size.
 * Infinities and NaN: a token's key and value show in no row before it, a cached one's in its own sequence and head only.  w, beta, log_f and c have to be
 * finite: one that is not may spoil all rows and keys of its sequence and head.
 * workspace: path_paged_workspace_bytes(...) bytes (0 for arguments that the calls reject; grows with every bound, so that one for the largest call serves
 * all smaller ones; path_paged_append as with group 1), 256-byte aligned; contents undefined before and after.
 * Errors: PATH_ERR_SHAPE for nseq, H, group or max_new < 1, group > 64, T or max_cached < 0, a page size that is not allowed, or max_cached >
 * pages_per_seq * page_size, more than 65535 of nseq * H or H * group, or bounds for which a kernel would need 2^32 threads (fp32: T * H * group of 2^26;
 * bf16: 2^28; thousands of sequences times heads with bounds of millions of cached tokens); PATH_ERR_NULL also if only one of log_f and cpages is given.  T = 0 does nothing.
 */
size_t path_paged_workspace_bytes(int nseq, int T, int max_new, int max_cached, int H, int group, int d, path_dtype_t dt);
path_status_t path_paged_attn(const void* q, const void* k, const void* v, const void* w, const void* beta, const void* log_f,
                              const void* kpages, const void* vpages, const float* cpages, const int* page_table,
                              const int* cached, const int* cu_new, void* o, float* lse, int nseq, int T, int max_new,
                              int max_cached, int num_pages, int page_size, int pages_per_seq, int H, int group, int d,
                              float scale, path_dtype_t dt, void* workspace, size_t workspace_bytes, void* stream);
path_status_t path_paged_append(const void* k, const void* v, const void* w, const void* beta, const void* log_f,
                                void* kpages, void* vpages, float* cpages, const int* page_table, const int* cached,
                                const int* cu_new, int nseq, int T, int max_new, int max_cached, int num_pages,
                                int page_size, int pages_per_seq, int H, int d, path_dtype_t dt, void* workspace,
                                size_t workspace_bytes, void* stream);
path_status_t path_paged_extend(const void* q, const void* k, const void* v, const void* w, const void* beta, const void* log_f,
                                void* kpages, void* vpages, float* cpages, const int* page_table, const int* cached,
                                const int* cu_new, void* o, float* lse, int nseq, int T, int max_new, int max_cached,
                                int num_pages, int page_size, int pages_per_seq, int H, int group, int d, float scale,
                                path_dtype_t dt, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Page tables of the path_paged_* calls, made to fit the requests' lengths on the GPU (lengths, tables and the stack of free pages are DEVICE int32 arrays; nothing is
 * read back, so a captured call follows them through its replays).  For every sequence, cached [nseq] is how many tokens stay and new_tokens [nseq] how many the coming call
 * brings (0 and 0: the sequence has ended; a smaller `cached` than before: drafts were dropped; negative counts as 0):
 *   1. entries of page_table [nseq, pages_per_seq] behind the ceil((cached + new) / page_size) pages that its tokens want go back: entries that are pages (0 .. num_pages - 1) are
 *      put on the stack free_pages [num_pages], whose first free_count [1] entries are free; all of them become -1.
 *   2. entries of new tokens' pages -- from ceil(cached / page_size) on -- that are no page get the one on top of the stack; if it is empty they become -1 (a hole) and are
 *      counted in missing [nseq].  Entries of pages that already hold cached tokens are left as they are.
 *   3. cu_new [nseq + 1] = offsets of the packed new tokens; slots [T] (64 bits; for caches of the caller's own beside these: the path_paged_* calls read the table, and path_delta_extend's slots are another thing) =
 *      page * page_size + place in it of every new token; -1 where there is no page, and for t behind
 *      the last new token.  T bounds the new tokens: offsets end at it, and tokens behind it take no part.  Tokens past pages_per_seq * page_size get no slot.
 * Pages go back before any is taken, both in the order of the table (sequence after sequence): the result is always the same.  A page is in one entry only (a page in two
 * entries goes back twice); what finds no room on the stack is dropped.  free_count outside 0 .. num_pages is held to it.
 * workspace: path_paged_plan_workspace_bytes(...) bytes (0 for sizes that are refused), 256-byte aligned.
 * Errors: PATH_ERR_SHAPE for nseq, num_pages or pages_per_seq < 1, T < 0, more than 2^22 sequences, or a page size that the path_paged_* calls do not take.  slots may be NULL if T = 0.
 */
size_t path_paged_plan_workspace_bytes(int nseq, int pages_per_seq, int T);
path_status_t path_paged_plan(const int* cached, const int* new_tokens, int* page_table, int* free_pages, int* free_count, int* cu_new, long long* slots, int* missing, int nseq,
                              int T, int num_pages, int page_size, int pages_per_seq, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Gated delta rule: the recurrence whose transitions PaTH attention takes into the softmax, as layers beside it use it.  A value head's state S [d, d] (rows: key index,
 * columns: value index; always fp32) follows
 *     S' = f_t S,   u_t = beta_t (v_t - S'^T k_t),   S = S' + k_t u_t^T,   o_t = scale S^T q_t,        f_t = exp(log_f_t),
 * evaluated by chunks of 64 tokens (served sequences of up to 8 new tokens: token by token).  H key heads, V = H * group value heads: value heads h * group .. h * group + group - 1
 * share q and k of head h.  log_f NULL: no gates.  q, k as given (unit vectors keep the recurrence from growing), beta as given.
 * Shapes: q, k, dq, dk [B,H,L,d], v, o, d_o, dv [B,V,L,d], beta, log_f, dbeta, dlog_f [B,V,L] (PATH_LAYOUT_BHLD), or the same with the token axis before the heads
 * (PATH_LAYOUT_BLHD), with nseq = B, max_len = L, T = B * L, cu_seqlens NULL; or packed: [T,H,d], [T,V,d], [T,V] (PATH_LAYOUT_BLHD), sequence s being the tokens
 * cu_seqlens[s] .. cu_seqlens[s+1]-1 (DEVICE int32 [nseq + 1], not decreasing), none longer than max_len; offsets and lengths past T and max_len are held to them.  Rows that belong to no sequence are left
 * as they are.  Sequences of no tokens: allowed, T = 0 too (pointers to tokens may be NULL then).
 *   path_delta_fwd        o; state_in [nseq,V,d,d] = first states (NULL: zeros), state_out = last ones (NULL: not wanted; may be state_in).
 *   path_delta_train_fwd  the same, leaving in `workspace` what the gradients need.
 *   path_delta_train_bwd  gradients of sum(d_o * o) + sum(d_state_out * state_out) (d_state_out NULL: zeros), from the workspace of path_delta_train_fwd on the same
 *                         tensors and sizes (state_in given to both or neither), as often as wanted; dlog_f is NULL exactly if log_f is, d_state_in if state_in is.  What a step
 *                         does not want to keep it recomputes by calling path_delta_train_fwd again.
 *   path_delta_extend     serving: packed new tokens (as cu_new of the path_paged_* calls, at most max_new a sequence) for states in a pool [num_slots,V,d,d], carried on in place.
 *                         slots [nseq] (DEVICE int32): the sequence's state; outside 0 .. num_slots - 1: starts from zeros and is not kept.  cached [nseq] (DEVICE int32, as in the
 *                         path_paged_* calls): tokens before these; 0: starts from zeros whatever the slot holds.  No new tokens: the slot is left as it is.  Two sequences of one call
 *                         have different slots (the state of one that is named twice is undefined; no fault).  A state moves on over every token of the call: where drafts may be dropped, the caller copies the state
 *                         before, or takes the drafts once they stay.
 * Arithmetic: PATH_F32 in 32 bits throughout.  PATH_BF16: states and sums in fp32, products of fp16 operands.  q and k are operands as they are (below 65504 in magnitude, as scale q.k has to
 * be; in steps of 2^-24); what comes of v, d_o and the states is held over a power of two per sequence, head and 16 value indices, chosen from the largest finite value of the first state and of the first chunk that is not all zeros, as the sum of two
 * fp16 numbers: states are off by some 1e-6 of their size, o and the 16-bit gradients by their own rounding and little more; o has the same bits whether states are handed out or not.  With beta near 2 over near-equal keys,
 * where a chunk's steps cancel, the error grows with their number: states to 1e-4 at 64 equal keys and beta = 2, and where nothing is forgotten it adds up from chunk to chunk (to 1e-3, and 4e-2 of
 * the gradients, after ten such chunks; PATH_F32 too: the matrices of such a chunk are nearly singular to 32 bits).  What the gradients of a chunk start from (its state, the gradient behind it, E and Y of its tokens) is kept
 * as one fp16 number each: before they are rounded dq, dk, dv and dbeta are off by up to 8e-4 of their norm, dlog_f, in which such sums cancel, by 2e-3 (keys whose products are 0.95), and all of them by up to 2^-4 of their largest
 * (dlog_f 2^-3) where the tokens of a chunk have one key, beta = 2 and values that alternate, in a state 3000 times their size. A sequence in which
 * anything outgrows that (1000 times; 64 times where gradients are wanted) is walked again over the largest value of all its chunks, then with 2^8 and 2^16 times the room.  Values
 * below 2^-19 of the largest lose bits, below 2^-30 they are lost (in the gradients but dv by the head's largest, and where two such meet sooner).  Keys longer than unit vectors with beta |k|^2 > 2 grow without bound, and past that come out infinite or NaN.
 * log_f below -200 counts as -200; log_f > 0 is carried as it is.  The matrices of a chunk end with fp16's smallest step, 2^-24 (PATH_BF16): where a run of tokens within a chunk adds up to s > 0, states are off by up to
 * 5 * 2^-25 e^s of the largest they get to, and from s = 11 on infinities and NaN may come out.
 * Infinities and NaN: by chunks, values that are not finite may spoil every row of the chunk of 64 tokens that they are in, and all later ones (gradients: all earlier ones too), of their
 * sequence and head; token by token, no row before them.
 * No atomics: the same bits every time.  Outputs overlap no input (state_out may be state_in).
 * workspace: path_delta_workspace_bytes(...) bytes (0 for sizes that are refused; training != 0 for the path_delta_train_* pair), 256-byte aligned; grows with every argument, so that one for the
 * largest call serves all smaller ones.
 * Errors: PATH_ERR_SHAPE for nseq, max_len, H or group < 1, T < 0, T != nseq * max_len without cu_seqlens, nseq * V > 2^19, (T / 64 + nseq) * V >= 2^23, V > 65535;
 * PATH_ERR_UNSUPPORTED for scale <= 0 or a packed batch that is not PATH_LAYOUT_BLHD; PATH_ERR_ALIGN for q, k, v, o, states or gradients of these off 16 bytes.
 */
size_t path_delta_workspace_bytes(int nseq, int T, int max_len, int H, int group, int d, path_dtype_t dt, int training);
path_status_t path_delta_fwd(const void* q, const void* k, const void* v, const void* beta, const void* log_f, const int* cu_seqlens, const float* state_in, void* o,
                             float* state_out, int nseq, int T, int max_len, int H, int group, int d, int layout, float scale, path_dtype_t dt, void* workspace,
                             size_t workspace_bytes, void* stream);
path_status_t path_delta_train_fwd(const void* q, const void* k, const void* v, const void* beta, const void* log_f, const int* cu_seqlens, const float* state_in, void* o,
                                   float* state_out, int nseq, int T, int max_len, int H, int group, int d, int layout, float scale, path_dtype_t dt, void* workspace,
                                   size_t workspace_bytes, void* stream);
path_status_t path_delta_train_bwd(const void* q, const void* k, const void* v, const void* beta, const void* log_f, const int* cu_seqlens, const float* state_in, const void* d_o,
                                   const float* d_state_out, void* dq, void* dk, void* dv, void* dbeta, void* dlog_f, float* d_state_in, int nseq, int T, int max_len,
                                   int H, int group, int d, int layout, float scale, path_dtype_t dt, void* workspace, size_t workspace_bytes, void* stream);
path_status_t path_delta_extend(const void* q, const void* k, const void* v, const void* beta, const void* log_f, float* states, const int* slots, const int* cached,
                                const int* cu_new, void* o, int nseq, int T, int max_new, int num_slots, int H, int group, int d, float scale, path_dtype_t dt, void* workspace,
                                size_t workspace_bytes, void* stream);

/*
 * Sequence-parallel forward: ONE device's share of the ring of paper Sec. 3.5 ("context parallelism": the
 * sequence is split into contiguous segments, one per device; a device attends its own segment, then the
 * segments to its left one hop at a time, applying one d x d product per super-block it has passed).  The three
 * calls below are what a device runs; moving the earlier segments' tiles between devices is the caller's
 * business (on one GPU a test walks the segments in turn).  [B,H,L,d] layout, forward only; plain PaTH, or
 * PaTH-FoX with the gates of each segment given to its own path_attn_ring_local (log_f [B,H,L], NULL = plain).
 *
 *   path_attn_ring_local   the device's own segment (L tokens, causal inside it): chunk transform, second level
 *                          and sweep.  Leaves in `state` (path_attn_ring_state_bytes(B,H,L,d) bytes, 16-byte
 *                          aligned, caller-owned device memory) what the sweep holds per query -- the query state,
 *                          now carried to the segment's left edge, the unnormalised output, the running maximum
 *                          and row sum, all fp32 -- and in `workspace` (path_attn_workspace_bytes(B,H,L,d,dt,0))
 *                          the segment's tiles, which devices to the RIGHT need for their hops: the regions of
 *                          the second-level keys, the values and the super-block products (2 L d + ceil(L/1024) d^2
 *                          elements per head).
 *   path_attn_ring_hop     attends the Lq queries of `state` to every key of an EARLIER segment of Lk tokens,
 *                          given as the workspace path_attn_ring_local filled on that segment (same B, H, d, dt),
 *                          and carries the state across that segment.  (Not a workspace of another entry point: the
 *                          ordinary forward of up to 1024 tokens and training pairs leave the second level out where
 *                          nobody else reads it.)  Hops are made nearest segment first.  Lk
 *                          must be a multiple of 64 (PATH_ERR_SHAPE): only the last segment of a sequence may be
 *                          ragged, and it is nobody's earlier segment.  with_gates != 0: PaTH-FoX (the earlier
 *                          segment's gate sums are in its workspace; every segment of a sequence uses gates or none).
 *   path_attn_ring_finish  o = O / l, lse = m + log l from `state` (after the last hop; for the first segment
 *                          right after path_attn_ring_local).  PaTH-FoX: gates_workspace = the workspace of the
 *                          device's OWN path_attn_ring_local (it holds the segment's gate sums); NULL = plain.
 *
 * With segment lengths that are multiples of 1024 (the second blocking level) the result is bit-identical to
 * path_attn_fwd on the whole sequence: the same tiles, the same products in the same order, the state kept in
 * fp32 between the calls.  Other lengths differ from it by rounding only.  Errors as for path_attn_fwd.
 */
size_t path_attn_ring_state_bytes(int B, int H, int L, int d);
/* Byte offsets and lengths, inside a segment's workspace, of the four regions a hop reads (host arrays of 4):
 * [0] second-level keys, [1] values, [2] super-block products, [3] gate sums (PaTH-FoX only).  A device that
 * receives an earlier segment needs a buffer of path_attn_workspace_bytes(B,H,L,d,dt,0) bytes with these regions
 * filled; the rest of it is never read by path_attn_ring_hop. */
path_status_t path_attn_ring_regions(int B, int H, int L, int d, path_dtype_t dt, size_t offsets[4], size_t bytes[4]);
path_status_t path_attn_ring_local(const void* q, const void* k, const void* v, const void* w, const void* beta,
                                   const void* log_f, void* state, int B, int H, int L, int d, float scale,
                                   path_dtype_t dt, void* workspace, size_t workspace_bytes, void* stream);
path_status_t path_attn_ring_hop(void* state, int B, int H, int Lq, const void* remote_workspace,
                                 size_t remote_workspace_bytes, int Lk, int d, int with_gates, float scale,
                                 path_dtype_t dt, void* stream);
path_status_t path_attn_ring_finish(const void* state, void* o, float* lse, int B, int H, int L, int d,
                                    path_dtype_t dt, const void* gates_workspace, size_t gates_workspace_bytes,
                                    void* stream);

/*
 * Measurement aid, not part of the method: a register-resident chain of 32x32x16 fp16 MFMA products (four
 * independent accumulators per wave, `waves_per_simd` waves on each of the 1024 SIMDs, `iters` x 16 products
 * per wave, no memory traffic inside the loop) for calibrating "percent of peak" against what the matrix pipes
 * deliver at the clock they actually hold.  It enqueues one kernel on `stream`; the caller times it.  The work is
 * path_probe_mfma_flops(waves_per_simd, iters) floating-point operations.  `sink` is device memory of at least
 * 1024 * 4 * 64 * 4 bytes (one float per lane), written with values nobody needs.  waves_per_simd must be 1, 2
 * or 4 and iters >= 1 (else PATH_ERR_SHAPE).
 */
double path_probe_mfma_flops(int waves_per_simd, int iters);
path_status_t path_probe_mfma(void* sink, int waves_per_simd, int iters, void* stream);
/*
 * The same chain with a choice of operands.  random_operands = 0: smooth, slowly varying values (what
 * path_probe_mfma runs); != 0: fp16 values of random sign, random significand and magnitudes 0.25 .. 4, the kind
 * of operands the method's kernels multiply.  The products draw more power on those, the chip holds a lower
 * clock, and the rate drops from about 2.1 to about 1.6 PFLOP/s: the second figure is the practical ceiling of an
 * MFMA-bound kernel on real data.
 */
path_status_t path_probe_mfma_operands(void* sink, int waves_per_simd, int iters, int random_operands, void* stream);

/*
 * path_decode_step for callers that cannot allocate or pass scratch memory: code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc.  Same arguments, results (bit for bit) and error
 * codes as path_decode_step, minus the workspace: the per-split partial results go to a device array of
 * PATH_DECODE_STATIC_BYTES (8 MiB) that is part of the library's image -- every GPU the library runs on
 * holds one copy until the process ends.  The call allocates nothing (no hipMalloc / hipFree, no allocating
 * library routine); on its first use on a device it looks the array's address up once.
 *   Limit: path_decode_workspace_bytes(B, H, d) <= PATH_DECODE_STATIC_BYTES, i.e. B*H <= 252 at d = 128 and
 *   B*H <= 496 at d = 64; beyond it PATH_ERR_WORKSPACE (the reason is in path_attn_last_error()).
 *   All calls on one GPU share the one array, which keeps the previous call's contents (nothing in it has to
 *   start at zero: a split's record counts once it carries the call's own mark, or, of a captured call, in the second
 *   launch that merges them).  Calls that may overlap on one GPU -- different streams without an ordering between
 *   them, or several host threads -- RACE on it: order them.  (A race spoils the calls that overlap, not later ones.)
 * path_decode_static_scratch_bytes returns PATH_DECODE_STATIC_BYTES.
 */
#define PATH_DECODE_STATIC_BYTES (8u * 1024u * 1024u)
size_t path_decode_static_scratch_bytes(void);
path_status_t path_decode_step_static(const void* q, const void* k, const void* v, const void* w,
                                      const void* beta, void* kcache, void* vcache, int n, int Lmax,
                                      void* o, float* lse, int B, int H, int d, float scale,
                                      path_dtype_t dt, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PATH_ATTN_H */
