// Gated delta rule, token by token: up to DELTA_FEW new tokens of each sequence, for states in a pool.
//
// A workgroup has 32 columns of a head's state, a thread 4 of them in D / 32 successive rows: the state is read once and written once, 128 bytes of a row at a
// time, and stays in registers between the tokens.  For a token, S^T k and S^T q are summed over the rows together, f and k u^T put in afterwards:
// o = scale (f S^T q + (k.q) u): one exchange between the waves per token.  Everything in 32 bits.  Bound by the states' way from and to memory where they are many (64 sequences of 32
// heads, d = 128: 268 MB in 42 us, a part of it held by the last cache level), else by latency: 16 heads of one sequence 4.3 us, five tokens of 16 sequences' 256 heads 13.6.
#include "delta_decl.h"

namespace path {

template <typename T, int N> struct Few { T x[N]; };

template <typename T, int D>
__global__ __launch_bounds__(256) void delta_step_kernel(DeltaArgs a) {
    constexpr int NR = D / 32;      // rows of a thread
    __shared__ float sums[2][4][8][9];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, cq = tid & 7, r0 = (tid >> 3) * NR;
    const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x / (D / 32)), part = blockIdx.x - unit * (D / 32);
    const int s = __builtin_amdgcn_readfirstlane(unit / a.V), hv = unit - s * a.V, hk = __builtin_amdgcn_readfirstlane(hv / a.G);
    const DeltaSeq sq = delta_seq(a, s);
    if (sq.len < 1 || sq.len > a.few) return;
    const int col = part * 32 + 4 * cq, slot = a.slots[s];
    const bool held = slot >= 0 && slot < a.num_slots;
    float* const st = held ? a.states + ((size_t)slot * a.V + hv) * D * D + (size_t)r0 * D + col : nullptr;
    f32x4 S[NR];
    const bool old = held && a.cached[s] > 0;
#pragma unroll
    for (int i = 0; i < NR; ++i) S[i] = old ? *reinterpret_cast<const f32x4*>(st + i * D) : f32x4{0.f, 0.f, 0.f, 0.f};

    const long long kat = delta_at(a, sq, s, a.ks, a.kt) + hk * a.kh + r0, vat = delta_at(a, sq, s, a.vs, a.vt) + hv * a.vh + col, sat = delta_at(a, sq, s, a.ss, a.st) + hv * a.sh;
    const T *const kp = static_cast<const T*>(a.k) + kat, *const qp = static_cast<const T*>(a.q) + kat, *const vp = static_cast<const T*>(a.v) + vat;
    const T *const bp = static_cast<const T*>(a.beta) + sat, *const fp = a.log_f ? static_cast<const T*>(a.log_f) + sat : nullptr;
    T* const op = static_cast<T*>(a.o) + vat;
    struct Token { Few<T, NR> k, q; Few<T, 4> v; T be, lf; } tok;
    auto load = [&](int t) {
        Token x;
        x.k = *reinterpret_cast<const Few<T, NR>*>(kp + t * a.kt);
        x.q = *reinterpret_cast<const Few<T, NR>*>(qp + t * a.kt);
        x.v = *reinterpret_cast<const Few<T, 4>*>(vp + t * a.vt);
        x.be = bp[t * a.st];
        x.lf = fp ? fp[t * a.st] : (T)0.f;
        return x;
    };
    tok = load(0);
    for (int t = 0; t < sq.len; ++t) {
        const Token x = tok;
        if (t + 1 < sq.len) tok = load(t + 1);
        float k[NR], q[NR], y[9];      // S^T k, S^T q, k.q
        f32x4 p = {0.f, 0.f, 0.f, 0.f}, z = p;
        y[8] = 0.f;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            k[i] = (float)x.k.x[i];
            q[i] = (float)x.q.x[i];
            p += S[i] * k[i];
            z += S[i] * q[i];
            y[8] += k[i] * q[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) { y[i] = p[i]; y[4 + i] = z[i]; }
#pragma unroll
        for (int b = 8; b < 64; b *= 2)
#pragma unroll
            for (int i = 0; i < 9; ++i) y[i] += __shfl_xor(y[i], b);
        float(*const mine)[8][9] = sums[t & 1];      // (a wave is at most one token ahead of another)
        if (lane < 8)
#pragma unroll
            for (int i = 0; i < 9; ++i) mine[wv][cq][i] = y[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 9; ++i) y[i] = (mine[0][cq][i] + mine[1][cq][i]) + (mine[2][cq][i] + mine[3][cq][i]);
        const float f = expf((float)x.lf), be = (float)x.be;
        f32x4 u;
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = be * ((float)x.v.x[i] - f * y[i]);
        if (r0 == 0) {
            Few<T, 4> o;
#pragma unroll
            for (int i = 0; i < 4; ++i) o.x[i] = (T)(a.scale * (f * y[4 + i] + y[8] * u[i]));
            *reinterpret_cast<Few<T, 4>*>(op + t * a.vt) = o;
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) S[i] = S[i] * f + u * k[i];
    }
    if (held)
#pragma unroll
        for (int i = 0; i < NR; ++i) *reinterpret_cast<f32x4*>(st + i * D) = S[i];
}

template <typename T, int D> static hipError_t launch(const DeltaArgs& a, hipStream_t stream) {
    delta_step_kernel<T, D><<<dim3((unsigned)a.nseq * a.V * (D / 32)), dim3(256), 0, stream>>>(a);
    return hipGetLastError();
}
hipError_t launch_delta_step(const DeltaArgs& a, int d, int is_bf16, hipStream_t stream) {
    if (is_bf16) return d == 64 ? launch<bf16_t, 64>(a, stream) : launch<bf16_t, 128>(a, stream);
    return d == 64 ? launch<float, 64>(a, stream) : launch<float, 128>(a, stream);
}

}  // namespace path
