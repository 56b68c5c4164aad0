// Gated delta rule: what host code and the kernels of delta_*.hip share.
//
// A value head's state S [d, d] (rows: key index, columns: value index) follows
//   S' = f_t S,  u_t = beta_t (v_t - S'^T k_t),  S = S' + k_t u_t^T,  o_t = scale S^T q_t,   f_t = exp(log_f_t).
// By chunks of 64 tokens, b the running sums of log f inside the chunk, gamma = exp(b), rho_i = exp(b_63 - b_i), D_ri = exp(b_r - b_i) for i <= r (every
// exponent that is formed is that of a difference, at most 0 for gates that forget):
//   L = strictLower(D o K K^T),  M = scale lower(D o Q K^T),  P = (I + L diag(beta))^-1,  A = (I + diag(beta) L)^-1 = I - diag(beta) P L        (delta_prep.hip, all chunks at once)
//   E = P (V - diag(gamma) K S),  U = diag(beta) E,  O = scale diag(gamma) Q S + M U,  S <- gamma_63 S + K^T diag(rho) U          (delta_scan.hip, chunk after chunk)
// and the gradients, G that of the state behind the chunk:
//   dU = M^T dO + diag(rho) K G,  Y = A^T dU,  dV = diag(beta) Y,  G <- gamma_63 G + Q^T diag(scale gamma) dO - K^T diag(gamma beta) Y     (delta_scan.hip, backwards)
//   dbeta_r = Y_r.E_r,  X = Y U^T,  N = dO U^T,  Gq = scale lower(N o D),  Gk = -strictLower(diag(beta) X o D)
//   dQ = Gq K + scale diag(gamma) dO S^T,   dK = Gk K - diag(gamma beta) Y S^T  +  Gk^T K + Gq^T Q + diag(rho) U G^T     ("read" and "written" part)
//   dlog_f_t = sum_{r >= t} (q_r.dq_r + k_r.dk_r(read) - k_r.dk_r(written)) + gamma_63 <S, G> + sum_i rho_i k_i.(U G^T)_i                      (delta_grad.hip)
// (E: what a token's prediction is off.  U = A diag(beta) (..) is the same, but leaves no E, which dbeta needs, where beta is 0.)
#pragma once
#include "path_common.h"

namespace path {

constexpr int DELTA_FEW = 8;       // a sequence with up to so many new tokens is taken token by token (served calls)
constexpr int DELTA_CUT = 36;      // sequences of so many chunks are cut into segments where heads are few
constexpr int DELTA_ROWS = 5;      // numbers kept per token between the kernels: beta, gamma, rho, b rounded to 32 bits, and what that rounding left

struct DeltaArgs {
    const void *q, *k, *v, *beta, *log_f;      // log_f NULL: no gates
    void* o;
    const int* cu;                             // NULL: sequences of one length
    const float* state_in;                     // [nseq, V, d, d]; NULL: zeros
    float* state_out;                          // NULL: not wanted
    float* states;                             // served calls: the pool, slots, and which sequences start afresh
    const int *slots, *cached;
    int num_slots;
    int nseq, T, L, H, G, V, NC, tiles;        // V = H * G value heads; NC chunks of the longest sequence; tiles: chunks reserved for all sequences
    int few;                                   // sequences of up to `few` tokens are not the chunk kernels'
    long long ks, kt, kh, vs, vt, vh, ss, st, sh;      // element strides of sequence, token and head: q, k; v, o; beta, log_f
    float scale;
    int nseg, seg;                             // segments of the longest sequence, chunks of a segment (outputs alone; 1: sequences are not cut)
    float* parts;                              // [nseq * V][nseg - 1][2][d][d]: what the segments do to a state
    void *p, *m, *at, *mt;                     // per (tile, head): P and M as operand fragments; training: the transposes of A and M
    float* rows;                               // per (tile, head): [DELTA_ROWS][64]
    // training: per (tile, head) the state before the chunk and the gradient behind it, [value index][key index], E and Y, [value index][token]: fp32 in rows, or fp16, over the powers of two that the scans
    // chose per (sequence, head) and 16 value indices, in fragments of 16 value indices by 32: [d / 16][d / 32 or 2][lane][8]
    void *sm, *gm, *em, *ym;
    int *vex, *gex;                            // [nseq * V][8]: of S and E, of G and Y
    const void* d_o;
    const float* d_state;                      // gradient of the last states; NULL: zeros
    void *dq, *dk, *dv, *dbeta, *dlog_f;
    float* d_state_in;
};

// The sequence's length, its first chunk's number among the tiles, and where its tokens start in tensors of the given strides.  Offsets outside
// the packed tensors are held to them.  A packed batch's sequence s has the tiles from start / 64 + s on: no two share one, and there are at most T / 64 + nseq.
struct DeltaSeq { int len, tile0; long long start; };
__device__ __forceinline__ int delta_held(int x, int T) { return x < 0 ? 0 : x > T ? T : x; }
__device__ __forceinline__ DeltaSeq delta_seq(const DeltaArgs& a, int s) {
    if (!a.cu) return {a.L, s * a.NC, 0};
    const int b = delta_held(a.cu[s], a.T), e = delta_held(a.cu[s + 1], a.T);
    const int n = e - b;
    return {n < 0 ? 0 : n > a.L ? a.L : n, b / CHUNK + s, b};
}
__device__ __forceinline__ long long delta_at(const DeltaArgs& a, const DeltaSeq& q, int s, long long seq, long long tok) {
    return a.cu ? q.start * tok : s * seq;
}
// Sequence and chunk of a tile (a whole wave asks); false: the tile is nobody's, or its sequence is short.
__device__ __forceinline__ bool delta_tile(const DeltaArgs& a, int tile, int lane, int& s, int& c, DeltaSeq& q) {
    if (!a.cu) {
        s = __builtin_amdgcn_readfirstlane(tile / a.NC);
    } else {
        // the last sequence whose first tile is not behind this one, by 64 probes at a time: two reads that wait for one another for up to 4096 sequences
        int lo = 0, n = a.nseq, step = 1;
        do {
            step = (n + 63) / 64;
            const int i = lo + lane * step;
            const bool before = lane * step < n && delta_held(a.cu[lane * step < n ? i : lo], a.T) / CHUNK + i <= tile;
            const int k = __popcll(__ballot(before)), at = k > 0 ? (k - 1) * step : 0;
            lo += at;
            n = n - at < step ? n - at : step;
        } while (step > 1);
        s = lo;
    }
    q = delta_seq(a, s);
    c = tile - q.tile0;
    return c >= 0 && (long long)c * CHUNK < q.len && q.len > a.few;
}

hipError_t launch_delta_prep(const DeltaArgs& a, int d, int is_bf16, bool training, hipStream_t stream);
hipError_t launch_delta_scan(const DeltaArgs& a, int d, int is_bf16, int mode, hipStream_t stream);      // 0: o; 1: o, and what the backward needs; 2: backwards
int delta_segments(long long units, int d, int is_bf16, long long chunks);
hipError_t launch_delta_grad(const DeltaArgs& a, int d, int is_bf16, hipStream_t stream);
hipError_t launch_delta_step(const DeltaArgs& a, int d, int is_bf16, hipStream_t stream);

}  // namespace path
