// Gated delta rule: the states, chunk after chunk, and backwards their gradients (delta_decl.h has the formulas).
//
// A workgroup has CT * 16 columns (value indices) of a head's state.  Four waves carry it on, each a quarter of its rows (key indices), in registers, and of a chunk's products
// with it the 16 tokens of one result tile; four more do what the chain of chunks does not wait for: the outputs (forward), and what d_o adds to dU and to the state's
// gradient (backwards, a chunk ahead).  What one wave alone needs of K, Q, A and M comes from memory straight into its registers, a chunk ahead; what others need -- the
// state, the predictions' errors, U -- is exchanged through LDS as operands, split once.  Three barriers a chunk.
//
// Bound by the latency of a chunk: two exchanges and four products that wait for one another.  d = 128, 64 heads of 8192 tokens, 32 columns: 302 us, 2.3 a chunk, 2.4 TB/s of its own traffic
// (738 MB: K, Q, V, P, M in, o out); with what the backward needs 380 us (1.14 GB), backwards 363 us (1.0 GB).  Of the way there, with operands of one part, which take 211 us: one wave per 16 columns, without exchanges
// (64 dependent products a chunk), 465 us, four waves for everything, over bf16 operands in more parts, 331, four more for the outputs and fp16 operands 256; loads one chunk ahead instead of two 262.
#include <type_traits>

#include "delta_parts.h"

namespace path {

enum { DELTA_O = 0, DELTA_KEEP = 1, DELTA_BACK = 2, DELTA_PART = 3 };      // forward; forward that keeps what the backward needs; backwards; what segments do to a state

template <typename T> struct DeltaOperand { typedef T type; };
template <> struct DeltaOperand<bf16_t> { typedef half_t type; };

template <typename T, int D, int CT, int MODE>
struct ScanLds {
    typedef typename DeltaOperand<T>::type C;
    typedef DeltaOps<C> P;
    static constexpr int NP = P::NP, NS = D / P::SL, CS = 64 / P::SL;                      // slabs of the state's rows, of a chunk
    static constexpr int TW = D / 64;                                          // state tiles of a wave
    static constexpr bool BACK = MODE == DELTA_BACK, HALF = sizeof(T) == 2;
    // exchange areas: state; predictions' errors (dU); diag(rho) U, U (the operand of the gradient's update, and Y to be kept); forward E, to be kept; backwards d_o
    // and diag(gamma) d_o as operands, and what they add up to, in fp32
    static constexpr int AREA = CS * NP * CT * 1024, S = 0, Y = S + NS * NP * CT * 1024, U = Y + AREA, V = U + AREA, O = V + AREA, OG = O + (MODE == DELTA_KEEP || BACK ? CS * CT * 1024 : 0);
    static constexpr int DU = OG + (BACK ? AREA : 0), DG = DU + (BACK ? 4 * CT * 1024 : 0), X = DG + (BACK ? 4 * TW * CT * 1024 : 0);
    // K and the tokens' numbers, two chunks; a wave's own tokens of V (16-bit), its own columns of Q (backwards)
    static constexpr int KT = X + 256, NUM = KT + 2 * DeltaTile<C, D>::BYTES, VT = NUM + 2 * 768, QT = VT + (HALF ? (BACK ? 8 : 4) * CT * 512 : 0);
    static constexpr int SW = HALF ? 32 : 16 * TW, SROW = HALF ? 64 : (SW + 4) * 4;      // columns of Q: elements, bytes of a row
    static constexpr int BYTES = QT + (BACK ? 4 * 64 * SROW : 0);
};

// `rows` rows of `row` bytes as a buffer, and what a lane loads from and stores to it
__device__ __forceinline__ __amdgpu_buffer_rsrc_t delta_buffer(const char* base, int rows, unsigned row) {
    const unsigned long long p = reinterpret_cast<unsigned long long>(base);
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)p), hi = __builtin_amdgcn_readfirstlane((unsigned)(p >> 32));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((unsigned long long)hi << 32 | lo), 0, __builtin_amdgcn_readfirstlane((rows < CHUNK ? rows : CHUNK) * row), 0x00020000);
}
template <typename F> __device__ __forceinline__ F delta_load16(__amdgpu_buffer_rsrc_t r, unsigned at) { return __builtin_bit_cast(F, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0)); }
template <typename T> __device__ __forceinline__ T delta_load1(__amdgpu_buffer_rsrc_t r, unsigned at) {
    if constexpr (sizeof(T) == 2) return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b16(r, at, 0, 0));
    else return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0));
}
template <typename T> __device__ __forceinline__ void delta_store4(__amdgpu_buffer_rsrc_t r, unsigned at, f32x4 x) {
    typedef unsigned u2 __attribute__((ext_vector_type(2)));
    typedef unsigned u4 __attribute__((ext_vector_type(4)));
    if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u2, __builtin_convertvector(x, bf16x4)), r, at, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, x), r, at, 0, 0);
}

// A packed batch's sequences in the order of their lengths, longest first (up to 64 of them; a whole wave asks): a long one that starts last would keep a few CUs busy alone.  16 heads of nine sequences
// of 40 to 2999 tokens: 238 us in their own order, 212 in this (backwards 222, 198; both before what is kept went out as fragments).
__device__ __forceinline__ int delta_longest(const DeltaArgs& a, int turn, int lane) {
    if (!a.cu || a.nseq == 1 || a.nseq > 64) return turn;
    const int len = delta_seq(a, lane < a.nseq ? lane : 0).len;
    int before = 0;
    for (int i = 0; i < a.nseq; ++i) {
        const int x = __builtin_amdgcn_readlane(len, i);
        before += x > len || (x == len && i < lane);
    }
    return __builtin_ctzll(__ballot(lane < a.nseq && before == turn));
}

template <typename T, int D, int CT, int MODE>
__global__ __launch_bounds__(512, 1) void delta_scan_kernel(DeltaArgs a) {
    typedef typename DeltaOperand<T>::type C;
    typedef DeltaOps<C> P;
    typedef typename P::Frag Frag;
    typedef decltype(delta_operand(typename Tr<T>::Frag())) Operand;
    typedef typename Tr<T>::Frag UserFrag;
    typedef ScanLds<T, D, CT, MODE> L;
    constexpr int NP = P::NP, NS = L::NS, CS = L::CS, TW = L::TW, ES = sizeof(T);
    constexpr bool BACK = MODE == DELTA_BACK, HALF = ES == 2;
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    // With few heads a sequence is cut into segments of `seg` chunks.  A segment does S -> A S + B: one launch walks all but the last from zeros, for B (the first one from the given state,
    // whose copy it leaves in place of its A), and, of V = 0, from the unit matrix, for A; the next walks all at once, each from the state that those before it make.
    constexpr bool PART = MODE == DELTA_PART;
    const int nseg = MODE == DELTA_O ? a.nseg : PART ? a.nseg - 1 : 1, parts = D / 16 / CT;
    int unit, part;
    if (!xcd_deal(blockIdx.x >> 3, blockIdx.x & 7, parts * (PART ? 2 : 1), a.nseq * a.V * nseg, unit, part)) return;
    const int at_seg = __builtin_amdgcn_readfirstlane(unit % nseg);
    unit = __builtin_amdgcn_readfirstlane(unit / nseg);
    const bool linear = PART && part >= parts;      // (the one for A)
    if (linear) part -= parts;
    const int turn = __builtin_amdgcn_readfirstlane(unit / a.V), s = delta_longest(a, turn, threadIdx.x & 63);
    const int hv = unit - turn * a.V, hk = __builtin_amdgcn_readfirstlane(hv / a.G);
    const DeltaSeq sq = delta_seq(a, s);
    const int len = __builtin_amdgcn_readfirstlane(sq.len), tile0 = __builtin_amdgcn_readfirstlane(sq.tile0);
    if (a.slots && len <= a.few) return;
    const int all = (len + CHUNK - 1) / CHUNK, c0 = MODE == DELTA_O || PART ? at_seg * a.seg : 0;
    const bool last = MODE == DELTA_KEEP || BACK || all - c0 <= a.seg, cut = MODE == DELTA_O && all > a.seg;      // the sequence's last segment; it has others
    if (at_seg > 0 && c0 >= all) return;
    if (PART && last) return;
    const int NC = last ? all - c0 : a.seg;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};

    // the first state: of a pool's slot, given, or zeros
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
    float* const joint = MODE == DELTA_O || PART ? a.parts + ((size_t)s * a.V + hv) * (a.nseg - 1) * 2 * D * D : nullptr;      // per segment B, A
    if (PART && at_seg > 0) from = nullptr;
    if (PART) to = joint + ((size_t)at_seg * 2 + linear) * D * D;
    if (cut) from = joint + (at_seg > 0 ? 0 : D * D);      // (the given state itself may be overwritten by now)
    if (!last && !PART) to = nullptr;
    // Operands start at 2^6 at most and may grow to fp16's end; those that are kept for the gradients of a chunk to 2^12, which leaves their products a place there.  Where one went
    // past that, the sequence is walked again over the largest value of all its chunks, or, if that is what it had, with 2^8 or 2^16 times the room (states about keys
    // of length one move by 2 |v| a token at most).  If nothing helps, a value that came in was not finite, and the first powers that held the others stand.
    constexpr int ROOM = MODE == DELTA_KEEP || BACK ? 6 : 10;
    constexpr float END = MODE == DELTA_KEEP || BACK ? 4096.f : 65504.f;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wv = wave & 3, n = lane & 15, g = lane >> 4;
    const bool chain = wave < 4;
    const int col = 16 * part * CT + n;      // the lane's value index (and + 16)
    int attempt = 0, first_e[CT];
#pragma unroll
    for (int x = 0; x < CT; ++x) first_e[x] = 0;
    auto walk_again = [&](bool past) {      // all waves ask, behind their last chunk
        if constexpr (!HALF) return false;
        const bool any = __ballot(past) != 0;
        if (lane == 0) reinterpret_cast<int*>(smem + L::X)[32 + wave] = any;
        __syncthreads();
        int n = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) n |= reinterpret_cast<const int*>(smem + L::X)[32 + i];
        return __builtin_amdgcn_readfirstlane(n) != 0 && attempt++ < 3;
    };
    f32x4 S[TW][CT];
    float down[CT], up[CT];
    // an exchange area's fragment, slabs of one requested together (left to itself the compiler waits for each on its own), and one tile of a slab as operands into it
    auto frags = [&](int area, DeltaParts<C, NP> (&f)[CS][CT]) {
#pragma unroll
        for (int sl = 0; sl < CS; ++sl)
#pragma unroll
            for (int x = 0; x < CT; ++x)
#pragma unroll
                for (int p = 0; p < NP; ++p) f[sl][x].p[p] = *reinterpret_cast<const Frag*>(smem + area + ((sl * CT + x) * NP + p) * 1024 + lane * 16);
    };
    auto frag1 = [&](int area, int sl, int x, int np) { return *reinterpret_cast<const Frag*>(smem + area + (sl * CT + x) * np * 1024 + lane * 16); };
    auto put = [&](auto parts, int area, int tile, int x, const f32x4& v) {
        constexpr int N = decltype(parts)::value;
        if constexpr (!HALF) {
            *reinterpret_cast<f32x4*>(smem + area + (tile * CT + x) * 1024 + lane * 16) = v;
        } else {
            const DeltaSplit4<N> r(v);
#pragma unroll
            for (int p = 0; p < N; ++p)
                *reinterpret_cast<uint2*>(smem + area + (((tile >> 1) * CT + x) * N + p) * 1024 + lane * 16 + (tile & 1) * 8) = r.p[p];
        }
    };
    const std::integral_constant<int, NP> all_parts{};
    const std::integral_constant<int, 1> one_part{};

    // A chunk's rows of the caller's tensors as a buffer that ends behind the sequence's last one: rows behind it come in as zeros, and nothing is stored there.
    // (A store under a condition would have every later wait for a load wait for the store as well.)
    constexpr int PPR = L::SW * ES / 16, NK = PPR;      // 16-byte pieces of a slice's row; of a slice per lane
    const char* const kb = static_cast<const char*>(a.k) + (delta_at(a, sq, s, a.ks, a.kt) + hk * a.kh) * ES;
    const char* const qb = static_cast<const char*>(a.q) + (kb - static_cast<const char*>(a.k));
    const long long vat = (delta_at(a, sq, s, a.vs, a.vt) + hv * a.vh + 16 * part * CT) * ES;
    const char* const vb = static_cast<const char*>(BACK ? a.d_o : a.v) + vat;
    char* const ob = static_cast<char*>(BACK ? a.dv : a.o) + vat;
    const unsigned krow = (unsigned)a.kt * ES, vrow = (unsigned)a.vt * ES;
    // (Pointers to a chunk's rows and matrices move with the chunks: made anew by multiplications they took a fifth of a chunk's time.)
    auto buffer = [&](const char* p, unsigned row, int c) { return delta_buffer(p, len - c * CHUNK, row); };
    if (PART && linear && at_seg == 0) {
        for (int t = 0; chain && t < TW; ++t)
#pragma unroll
            for (int x = 0; x < CT; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const size_t at = (size_t)P::row(TW * wv + t, 4 * g + j) * D + col + 16 * x;
                    to[at] = from ? from[at] : 0.f;
                }
        return;
    }
    const int step = BACK ? -1 : 1, first = BACK ? NC - 1 : c0;
    auto after = [&](int c) { const int y = c + step; return y >= c0 && y < c0 + NC ? y : c; };      // (behind the last chunk: that one again)
    auto at_first = [&](const char* base, unsigned row) { return base + (long long)(first > 0 ? first : 0) * CHUNK * row; };
    const size_t unit0 = (size_t)(tile0 + (first > 0 ? first : 0)) * a.V + hv;
    constexpr int TRI = NP * P::NLOW * 1024;
    auto moved = [&](const char* p, int c, int to, long long bytes) { return p + (to == c ? 0 : step * bytes); };      // from chunk c to `to`
    // Loads are two chunks ahead, in two sets of registers that the chunks use in turn: memory under this load takes longer than a chunk.
    auto in_turn = [&](auto&& body) {
        for (int i = 0, c = first; i < NC; i += 2, c += 2 * step) {
            body(std::integral_constant<int, 0>{}, i, c);
            if (i + 1 < NC) body(std::integral_constant<int, 1>{}, i + 1, c + step);
        }
    };
    // a later segment's first state: S <- A S + B over the segments before it, in fp32; S as operands by way of the exchange areas
    auto joined = [&](bool holds) {
        for (int i = 1; i < at_seg; ++i) {
            const float* const B = joint + (size_t)i * 2 * D * D;
            const float* const A = B + D * D;
            if (holds) {
                f32x4 m[TW][D / 16];
#pragma unroll
                for (int t = 0; t < TW; ++t)
#pragma unroll
                    for (int z = 0; z < D / 16; ++z) m[t][z] = *reinterpret_cast<const f32x4*>(A + (size_t)P::row(TW * wv + t, n) * D + P::row(z, 4 * g));
                f32x4 y[TW][CT];
#pragma unroll
                for (int t = 0; t < TW; ++t)
#pragma unroll
                    for (int x = 0; x < CT; ++x) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) y[t][x][j] = B[(size_t)P::row(TW * wv + t, 4 * g + j) * D + col + 16 * x];
                        *reinterpret_cast<f32x4*>(smem + ((TW * wv + t) * CT + x) * 1024 + lane * 16) = S[t][x];
                    }
                __syncthreads();
#pragma unroll
                for (int z = 0; z < D / 16; ++z)
#pragma unroll
                    for (int x = 0; x < CT; ++x) {
                        const f32x4 b = *reinterpret_cast<const f32x4*>(smem + (z * CT + x) * 1024 + lane * 16);
#pragma unroll
                        for (int t = 0; t < TW; ++t) y[t][x] = DeltaOps<float>::mma(m[t][z], b, y[t][x]);
                    }
#pragma unroll
                for (int t = 0; t < TW; ++t)
#pragma unroll
                    for (int x = 0; x < CT; ++x) S[t][x] = y[t][x];
                __syncthreads();
            } else {
                __syncthreads();
                __syncthreads();
            }
        }
    };
    // The first state, and the powers of two of the columns: down for what comes in, up for what goes out.  They are those of the first state and of the first chunk that holds anything
    // but zeros (a look at all of V would read it twice); a sequence that outgrows them is walked again.
    auto begin = [&](bool holds) {      // (a wave of the first four holds a part of the state)
#pragma unroll
        for (int t = 0; t < TW; ++t)
#pragma unroll
            for (int x = 0; x < CT; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j) S[t][x][j] = holds && from ? from[(size_t)P::row(TW * wv + t, 4 * g + j) * D + col + 16 * x] : 0.f;
        if (PART && linear && at_seg > 0 && holds)
#pragma unroll
            for (int t = 0; t < TW; ++t)
#pragma unroll
                for (int x = 0; x < CT; ++x)
#pragma unroll
                    for (int j = 0; j < 4; ++j) S[t][x][j] = P::row(TW * wv + t, 4 * g + j) == col + 16 * x ? 1.f : 0.f;
        if (cut) joined(holds);
#pragma unroll
        for (int x = 0; x < CT; ++x) down[x] = up[x] = 1.f;
        if constexpr (HALF) {
            float* const xs = reinterpret_cast<float*>(smem + L::X);
            float m[CT], all[CT];
#pragma unroll
            for (int x = 0; x < CT; ++x) {
                all[x] = m[x] = 0.f;
                if (holds)
#pragma unroll
                    for (int t = 0; t < TW; ++t)
#pragma unroll
                        for (int j = 0; j < 4; ++j) m[x] = fmaxf(m[x], delta_finite(S[t][x][j]));
            }
            for (int i = 0, c = first; i < (NC > 0 ? NC : 1); ++i, c += step) {
                if (NC > 0 && wave < 2 * CT && !linear) {      // a piece of eight columns to a thread
                    const UserFrag f = delta_load16<UserFrag>(buffer(vb + (long long)c * CHUNK * vrow, vrow, c), tid / (2 * CT) * vrow + tid % (2 * CT) * 16);
                    float y = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) y = fmaxf(y, delta_finite((float)f[e]));
#pragma unroll
                    for (int x = 0; x < CT; ++x) m[x] = fmaxf(m[x], CT == 1 || (lane >> 1 & 1) == x ? y : 0.f);
                }
#pragma unroll
                for (int x = 0; x < CT; ++x) {
#pragma unroll
                    for (int z = 1; z < 64; z *= 2) m[x] = fmaxf(m[x], __shfl_xor(m[x], z));
                    if (lane == 0) xs[x * 8 + wave] = m[x];
                }
                __syncthreads();
                float any = 0.f;
#pragma unroll
                for (int x = 0; x < CT; ++x) {
#pragma unroll
                    for (int z = 0; z < 8; ++z) all[x] = fmaxf(all[x], xs[x * 8 + z]);
                    any = fmaxf(any, all[x]);
                }
                if (attempt == 0 && __builtin_amdgcn_readfirstlane(any > 0.f)) break;
                __syncthreads();
            }
#pragma unroll
            for (int x = 0; x < CT; ++x) {
                int e = __builtin_amdgcn_readfirstlane(delta_exponent(all[x]));
                if (attempt == 0) first_e[x] = e;
                else if (attempt < 3) e += 8 * (attempt - (e > first_e[x]));
                else if (e - first_e[x] <= ROOM) e = first_e[x];
                down[x] = delta_power(-e);
                up[x] = delta_power(e);
                if ((MODE == DELTA_KEEP || BACK) && tid == 0) (BACK ? a.gex : a.vex)[((size_t)s * a.V + hv) * 8 + part * CT + x] = e;
#pragma unroll
                for (int t = 0; t < TW; ++t) S[t][x] = S[t][x] * down[x];
            }
        }
    };
    const unsigned row_at = P::row(wv, n) * krow + 16 * g;
    const unsigned slice_at = lane / PPR * krow + (HALF ? 32 * (TW * wv >> 1) : 16 * TW * wv) * ES + lane % PPR * 16;
    typedef DeltaTile<C, D> Tile;
    typedef const __attribute__((address_space(1))) Frag GlobalFrag;
    constexpr int RS = D * ES / 64;                       // 64-byte pieces of a row: a fragment of one each; 16-byte pieces of 16 rows per lane
    constexpr int UPR = D * ES / 16;                      // 16-byte pieces of a row
    auto load_rows = [&](const char* p, int c, UserFrag* f) {            // fragments of the wave's tokens
        const auto r = buffer(p, krow, c);
#pragma unroll
        for (int sl = 0; sl < RS; ++sl) f[sl] = delta_load16<UserFrag>(r, row_at + sl * 64);
    };
    auto load_slice = [&](const char* p, int c, UserFrag* f) {           // all rows of the wave's columns
        const auto r = buffer(p, krow, c);
#pragma unroll
        for (int i = 0; i < NK; ++i) f[i] = delta_load16<UserFrag>(r, slice_at + i * (64 / PPR) * krow);
    };
    const int slice = L::QT + wv * 64 * L::SROW;
    auto store_slice = [&](const UserFrag* f) {
#pragma unroll
        for (int i = 0; i < NK; ++i) *reinterpret_cast<Operand*>(smem + slice + (i * 64 + lane) / PPR * L::SROW + (lane % PPR) * 16) = delta_operand(f[i]);
    };
    // a quarter of a chunk's K for everybody, and the tokens' beta, gamma and rho
    auto load_tile = [&](const char* p, const char* num, int c, UserFrag* f, f32x4& w) {
        const auto r = buffer(p, krow, c);
#pragma unroll
        for (int i = 0; i < RS; ++i) f[i] = delta_load16<UserFrag>(r, (16 * wv + (i * 64 + lane) / UPR) * krow + lane % UPR * 16);
        typedef const __attribute__((address_space(1))) f32x4 Global4;
        if (wv == 0) w = *(Global4*)scalar_base(num, (lane < 48 ? lane : 47) * 16);
    };
    auto store_tile = [&](int c, const UserFrag* f, const f32x4& w) {
        const int at = L::KT + (c & 1) * Tile::BYTES;
#pragma unroll
        for (int i = 0; i < RS; ++i) *reinterpret_cast<Operand*>(smem + at + Tile::piece(16 * wv + (i * 64 + lane) / UPR, lane % UPR)) = delta_operand(f[i]);
        if (wv == 0 && lane < 48) *reinterpret_cast<f32x4*>(smem + L::NUM + (c & 1) * 768 + lane * 16) = w;
    };
    auto numbers = [&](int c, int which) { return *reinterpret_cast<const f32x4*>(smem + L::NUM + (c & 1) * 768 + (which * 64 + P::row(wv, 4 * g)) * 4); };      // of the lane's four tokens
    auto used = [&](int sl) { return BACK ? P::up(wv, sl) : P::low(wv, sl); };
    auto load_tri = [&](const char* p, DeltaParts<C, NP>* f) {      // (without branches: a slab that is not used is the wave's first or last one again)
#pragma unroll
        for (int sl = 0; sl < CS; ++sl) {
            const int at = BACK ? P::up_at(wv, used(sl) ? sl : CS - 1) : P::low_at(wv, used(sl) ? sl : 0);
#pragma unroll
            for (int z = 0; z < NP; ++z) f[sl].p[z] = *(GlobalFrag*)scalar_base(p + (z * P::NLOW + at) * 1024, lane * 16);
        }
    };
    // The wave's tokens and columns of V (backwards: dO): 16-bit numbers by whole pieces, to the lane that takes four tokens of a column by way of LDS
    constexpr int VN = HALF ? 1 : 4 * CT;
    typedef typename std::conditional<HALF, UserFrag, float>::type Value;
    const int vt = L::VT + (BACK && !chain ? 4 * CT * 512 : 0) + wv * CT * 512;
    auto load_values = [&](const char* p, int c, Value (&v)[VN]) {
        const auto r = buffer(p, vrow, c);
        if constexpr (HALF) {
            if (lane < 32 * CT) v[0] = delta_load16<UserFrag>(r, P::row(wv, lane / (2 * CT)) * vrow + lane % (2 * CT) * 16);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int x = 0; x < CT; ++x) v[4 * x + j] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, P::row(wv, 4 * g + j) * vrow + (n + 16 * x) * 4, 0, 0));
        }
    };
    auto store_values = [&](const Value (&v)[VN]) {
        if constexpr (HALF)
            if (lane < 32 * CT) *reinterpret_cast<UserFrag*>(smem + vt + lane * 16) = v[0];
    };
    auto values = [&](const Value (&v)[VN], f32x4* V) {
#pragma unroll
        for (int x = 0; x < CT; ++x) {
            if constexpr (HALF) {
                const uint2 w = __builtin_bit_cast(uint2, delta_ld_tr(smem + vt + (4 * g + (n >> 2)) * CT * 32 + 32 * x + (n & 3) * 8));
                V[x] = f32x4{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u)} * down[x];
            } else {
                V[x] = f32x4{v[4 * x], v[4 * x + 1], v[4 * x + 2], v[4 * x + 3]};
            }
        }
    };
    // tiles [TW][CT] += (the wave's columns of K, or of Q)^T y; at: of row r, piece p of the matrix in LDS
    auto into = [&](f32x4 (&z)[TW][CT], const DeltaParts<C, NP> (&y)[CS][CT], auto at, int first_piece) {
#pragma unroll
        for (int sl = 0; sl < CS; ++sl)
#pragma unroll
            for (int t = 0; t < TW; ++t) {
                DeltaParts<C, 1> k;
                if constexpr (HALF) {
                    const unsigned char* const p = smem + at(8 * g + (n >> 2) + 32 * sl, first_piece + (n & 3)) + 8 * (TW == 2 ? t : wv & 1);
                    const halfx4 k0 = delta_ld_tr(p), k1 = delta_ld_tr(p + (at(4, 0) - at(0, 0)));
                    k.p[0] = halfx8{k0[0], k0[1], k0[2], k0[3], k1[0], k1[1], k1[2], k1[3]};
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) k.p[0][e] = *reinterpret_cast<const float*>(smem + at(16 * sl + 4 * g + e, first_piece + 4 * t + (n >> 2)) + (n & 3) * 4);
                }
#pragma unroll
                for (int x = 0; x < CT; ++x) z[t][x] = delta_mma(k, y[sl][x], z[t][x]);
            }
    };
    // the wave's tokens' rows of K times the state: tokens along the registers; of Q: tokens along the lanes
    auto times_state = [&](auto row, auto turned, f32x4* y) {
        constexpr int HS = NS * NP * CT > 16 ? NS / 2 : NS;      // slabs requested together: up to 64 registers
#pragma unroll
        for (int x = 0; x < CT; ++x) y[x] = zero;
#pragma unroll
        for (int s0 = 0; s0 < NS; s0 += HS) {
            DeltaParts<C, NP> f[HS][CT];
            DeltaParts<C, 1> q[HS];
#pragma unroll
            for (int sl = 0; sl < HS; ++sl) {
                q[sl].p[0] = row(s0 + sl);
#pragma unroll
                for (int x = 0; x < CT; ++x)
#pragma unroll
                    for (int p = 0; p < NP; ++p) f[sl][x].p[p] = *reinterpret_cast<const Frag*>(smem + L::S + (((s0 + sl) * CT + x) * NP + p) * 1024 + lane * 16);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int sl = 0; sl < HS; ++sl)
#pragma unroll
                for (int x = 0; x < CT; ++x) y[x] = decltype(turned)::value ? delta_mma(f[sl][x], q[sl], y[x]) : delta_mma(q[sl], f[sl][x], y[x]);
        }
    };
    // the wave's tokens' rows of P or M (transposed: of A^T or M^T) times y
    auto times = [&](const DeltaParts<C, NP>* m, const DeltaParts<C, NP> (&y)[CS][CT], auto turned, f32x4* o) {
#pragma unroll
        for (int sl = 0; sl < CS; ++sl)
            if (used(sl))
#pragma unroll
                for (int x = 0; x < CT; ++x) o[x] = decltype(turned)::value ? delta_mma(y[sl][x], m[sl], o[x]) : delta_mma(m[sl], y[sl][x], o[x]);
    };
    // A state's or token matrix's slabs to memory for the chunk's gradients; the waves take turns.  fp32: the lane's row of the transposed matrix; fp16: fragments as they are, 1 KB each, by value indices and
    // slabs (rows instead, of which a fragment has 64 bytes each, took 342 us where this took 300, both with operands of one part).
    auto keep = [&](void* out, int area, size_t u, int np, int slabs) {
        const int ld = slabs * P::SL;
        for (int sl = wv; sl < slabs; sl += 4)
#pragma unroll
            for (int x = 0; x < CT; ++x) {
                const size_t at = HALF ? (size_t)(((part * CT + x) * slabs + sl) * 64 + lane) * P::FE : (size_t)(col + 16 * x) * ld + P::SL * sl + P::FE * g;
                *reinterpret_cast<Frag*>(static_cast<C*>(out) + u * D * ld + at) = frag1(area, sl, x, np);
            }
    };
    auto put_state = [&]() {
#pragma unroll
        for (int x = 0; x < CT; ++x)
#pragma unroll
            for (int t = 0; t < TW; ++t) put(all_parts, L::S, TW * wv + t, x, S[t][x]);
    };

    const char *const ga = static_cast<const char*>(BACK ? a.at : a.p), *const gm = static_cast<const char*>(BACK ? a.mt : a.m);
    const long long dk = (long long)CHUNK * krow, dv = (long long)CHUNK * vrow, dtri = (long long)a.V * TRI, dnum = (long long)a.V * DELTA_ROWS * 256;      // bytes from chunk to chunk
    const std::true_type turned{};
    const std::false_type upright{};
    // Who brings K and the numbers: the waves that wait for the others
    constexpr bool CHAIN_STAGES = BACK;
    UserFrag kt[2][RS];
    f32x4 num[2];
    const char *kn, *nn;
    int kc;      // the chunk that they are at
    auto load_next = [&](UserFrag (&f)[RS], f32x4& w) {
        const int then = after(kc);
        kn = moved(kn, kc, then, dk);
        nn = moved(nn, kc, then, dnum);
        kc = then;
        load_tile(kn, nn, kc, f, w);
    };
    auto stage = [&](auto other, int next) {      // the next chunk's K, into the buffer that nobody has read since the last chunk's third barrier
        constexpr int O = decltype(other)::value;
        store_tile(next, kt[O], num[O]);
        load_next(kt[O], num[O]);
    };
    auto begin_tile = [&]() {
        if (NC == 0) return;
        kn = at_first(kb, krow);
        nn = reinterpret_cast<const char*>(a.rows) + unit0 * DELTA_ROWS * 256;
        kc = first;
        num[0] = num[1] = zero;
        load_tile(kn, nn, first, kt[0], num[0]);
        store_tile(first, kt[0], num[0]);
        load_next(kt[1], num[1]);
        load_next(kt[0], num[0]);
    };
    if (chain) for (;;) {
        begin(true);
        if (CHAIN_STAGES) begin_tile();
        float most_out = 0.f;
        DeltaParts<C, NP> A[2][CS];
        Value v[2][VN];
        const char *vn = at_first(vb, vrow), *an = ga + unit0 * TRI;
        int ahead = first;      // the chunk that they are at
        if (NC > 0) {
            // (in the order of the loop: waits for loads go by how many came after them)
            if (!BACK) load_values(vn, first, v[0]);
            load_tri(an, A[0]);
            ahead = after(first);
            vn = moved(vn, first, ahead, dv);
            an = moved(an, first, ahead, dtri);
            if (!BACK) load_values(vn, ahead, v[1]);
            load_tri(an, A[1]);
        }
        put_state();
        if (BACK && NC > 0) { lds_barrier(); lds_barrier(); lds_barrier(); }      // (the other waves' first chunk)
        in_turn([&](auto turn, int i, int c) {
            constexpr int T2 = decltype(turn)::value;
            const int next = after(c), then = after(ahead);
            f32x4 V[CT], y[CT];
            if (!BACK) {
                store_values(v[T2]);
                values(v[T2], V);
                vn = moved(vn, ahead, then, dv);
                load_values(vn, then, v[T2]);
            }
            lds_barrier();
            const int tile = L::KT + (c & 1) * Tile::BYTES;
            times_state([&](int sl) { return *reinterpret_cast<const Frag*>(smem + tile + Tile::piece(P::row(wv, n), 4 * sl + g)); }, upright, y);
            if (!BACK) {
                const f32x4 ga4 = numbers(c, 1);
#pragma unroll
                for (int x = 0; x < CT; ++x) put(all_parts, L::Y, wv, x, (PART && linear ? zero : V[x]) - ga4 * y[x]);
            } else {      // dU = diag(rho) K G + M^T dO
                const f32x4 rh = numbers(c, 2);
#pragma unroll
                for (int x = 0; x < CT; ++x) put(all_parts, L::Y, wv, x, y[x] * rh + *reinterpret_cast<const f32x4*>(smem + L::DU + (wv * CT + x) * 1024 + lane * 16));
            }
            lds_barrier();
            DeltaParts<C, NP> f[CS][CT];
            frags(L::Y, f);
            const f32x4 be = numbers(c, 0), w = numbers(c, BACK ? 1 : 2);
            const float g63 = *reinterpret_cast<const float*>(smem + L::NUM + (c & 1) * 768 + (64 + 63) * 4);
            __builtin_amdgcn_sched_barrier(0);
            f32x4 U[CT];
#pragma unroll
            for (int x = 0; x < CT; ++x) U[x] = zero;
            times(A[T2], f, upright, U);
#pragma unroll
            for (int x = 0; x < CT; ++x) {
                if (HALF)
#pragma unroll
                    for (int j = 0; j < 4; ++j) most_out = fmaxf(most_out, fmaxf(fabsf(U[x][j]), fabsf(be[j] * U[x][j])));
                if (!BACK) {      // (U: E at first)
                    if (MODE == DELTA_KEEP) put(one_part, L::O, wv, x, U[x]);
                    U[x] = be * U[x];
                    put(all_parts, L::U, wv, x, U[x] * w);
                    if (!PART) put(all_parts, L::V, wv, x, U[x]);
                } else {      // (U: the gradient's Y)
                    put(one_part, L::V, wv, x, U[x]);
                    U[x] = be * U[x];
                    put(all_parts, L::U, wv, x, -(w * U[x]));
                    if constexpr (!HALF) {      // dv, which with 16 bits the kernel of the chunks' gradients makes from Y
                        const auto r = buffer(ob + (long long)c * dv, vrow, c);
#pragma unroll
                        for (int j = 0; j < 4; ++j) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(U[x][j]), r, P::row(wv, 4 * g + j) * vrow + (n + 16 * x) * 4, 0, 0);
                    }
                }
            }
            lds_barrier();
            frags(L::U, f);
#pragma unroll
            for (int t = 0; t < TW; ++t)
#pragma unroll
                for (int x = 0; x < CT; ++x) {
                    S[t][x] = S[t][x] * g63;
                    if (BACK) S[t][x] = S[t][x] + *reinterpret_cast<const f32x4*>(smem + L::DG + ((TW * wv + t) * CT + x) * 1024 + lane * 16);
                }
            into(S, f, [&](int r, int p) { return tile + Tile::piece(r, p); }, HALF ? 4 * (TW * wv >> 1) : 4 * TW * wv);
            an = moved(an, ahead, then, dtri);
            load_tri(an, A[T2]);
            ahead = then;
            put_state();
            if (CHAIN_STAGES) stage(std::integral_constant<int, 1 - T2>{}, next);
        });
        bool past = most_out > END;
#pragma unroll
        for (int t = 0; t < TW; ++t)
#pragma unroll
            for (int x = 0; x < CT; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j) past |= (__float_as_uint(S[t][x][j]) & 0x7f800000u) == 0x7f800000u;
        if (walk_again(past)) continue;
        if (to) {
#pragma unroll
            for (int t = 0; t < TW; ++t)
#pragma unroll
                for (int x = 0; x < CT; ++x)
#pragma unroll
                    for (int j = 0; j < 4; ++j) to[(size_t)P::row(TW * wv + t, 4 * g + j) * D + col + 16 * x] = S[t][x][j] * up[x];
        }
        return;
    }
    if (PART) for (;;) {
        begin(false);
        begin_tile();
        in_turn([&](auto turn, int i, int c) {
            lds_barrier();
            lds_barrier();
            lds_barrier();
            stage(std::integral_constant<int, 1 - decltype(turn)::value>{}, after(c));
        });
        if (!walk_again(false)) return;
    }
    if (!BACK) for (;;) {
        begin(false);
        begin_tile();
        UserFrag Q[2][RS];
        Operand Qh[RS];
        DeltaParts<C, NP> M[2][CS];
        const char *qn = at_first(qb, krow), *mn = gm + unit0 * TRI;
        char* on = ob + c0 * dv;
        int ahead = first;
        if (NC > 0) {
            load_rows(qn, first, Q[0]);
            load_tri(mn, M[0]);
            ahead = after(first);
            qn = moved(qn, first, ahead, dk);
            mn = moved(mn, first, ahead, dtri);
            load_rows(qn, ahead, Q[1]);
            load_tri(mn, M[1]);
        }
        in_turn([&](auto turn, int i, int c) {
            constexpr int T2 = decltype(turn)::value;
            const int next = after(c), then = after(ahead);
            const size_t u = (size_t)(tile0 + c) * a.V + hv;
            f32x4 o[CT];
#pragma unroll
            for (int sl = 0; sl < RS; ++sl) Qh[sl] = delta_operand(Q[T2][sl]);
            qn = moved(qn, ahead, then, dk);
            load_rows(qn, then, Q[T2]);
            lds_barrier();
            times_state([&](int sl) { return Qh[sl]; }, turned, o);
            const float w = a.scale * *reinterpret_cast<const float*>(smem + L::NUM + (c & 1) * 768 + (64 + P::row(wv, n)) * 4);
            lds_barrier();
#pragma unroll
            for (int x = 0; x < CT; ++x) o[x] = o[x] * w;
            if (MODE == DELTA_KEEP) keep(a.sm, L::S, u, NP, NS);
            lds_barrier();
            DeltaParts<C, NP> f[CS][CT];
            frags(L::V, f);
            __builtin_amdgcn_sched_barrier(0);
            times(M[T2], f, turned, o);
            mn = moved(mn, ahead, then, dtri);
            load_tri(mn, M[T2]);
            ahead = then;
            if (MODE == DELTA_KEEP) keep(a.em, L::O, u, 1, CS);
            const auto r = buffer(on, vrow, c);
#pragma unroll
            for (int x = 0; x < CT; ++x) delta_store4<T>(r, P::row(wv, n) * vrow + (16 * x + 4 * g) * ES, o[x] * up[x]);
            on += dv;
            stage(std::integral_constant<int, 1 - T2>{}, next);
        });
        if (!walk_again(false)) return;
    }
    if (BACK) for (;;) {
        begin(false);
        float most_out = 0.f;
        if (NC > 0) {
        // Of the chunk that the first four waves come to next: M^T dO and Q^T diag(scale gamma) dO, in fp32.  The first goes out behind the second barrier (they have read
        // the one before), the second, held back, behind the first barrier of the next round.
        UserFrag qt[2][NK];
        DeltaParts<C, NP> M[2][CS];
        Value v[2][VN];
        f32x4 V[CT], du[CT], dg[TW][CT], ga4[2];
        auto gammas = [&](int c) {
            typedef const __attribute__((address_space(1))) f32x4 Global4;
            return *(Global4*)scalar_base(a.rows + (((size_t)(tile0 + c) * a.V + hv) * DELTA_ROWS + 1) * 64, P::row(wv, 4 * g) * 4);
        };
        const char *vn = at_first(vb, vrow), *qn = at_first(qb, krow), *mn = gm + unit0 * TRI;
        int ahead = first;
        load_values(vn, first, v[0]);
        load_slice(qn, first, qt[0]);
        ga4[0] = gammas(first);
        load_tri(mn, M[0]);
        ahead = after(first);
        vn = moved(vn, first, ahead, dv);
        qn = moved(qn, first, ahead, dk);
        mn = moved(mn, first, ahead, dtri);
        load_values(vn, ahead, v[1]);
        load_slice(qn, ahead, qt[1]);
        ga4[1] = gammas(ahead);
        load_tri(mn, M[1]);
#pragma unroll
        for (int t = 0; t < TW; ++t)
#pragma unroll
            for (int x = 0; x < CT; ++x) dg[t][x] = zero;
        // round i: this is at chunk i of theirs, they are at the one before
        auto round = [&](auto turn, int i, int c) {
            constexpr int T2 = decltype(turn)::value;
            const int then = after(ahead);
            const size_t u = (size_t)(tile0 + c - step) * a.V + hv;
            store_values(v[T2]);
            values(v[T2], V);
            vn = moved(vn, ahead, then, dv);
            load_values(vn, then, v[T2]);
            store_slice(qt[T2]);
            qn = moved(qn, ahead, then, dk);
            load_slice(qn, then, qt[T2]);
#pragma unroll
            for (int x = 0; x < CT; ++x) {
                if (HALF)
#pragma unroll
                    for (int j = 0; j < 4; ++j) most_out = fmaxf(most_out, fabsf(V[x][j]));
                put(one_part, L::O, wv, x, V[x]);
                put(all_parts, L::OG, wv, x, V[x] * (ga4[T2] * a.scale));
            }
            ga4[T2] = gammas(then);
            lds_barrier();
#pragma unroll
            for (int t = 0; t < TW; ++t)
#pragma unroll
                for (int x = 0; x < CT; ++x) *reinterpret_cast<f32x4*>(smem + L::DG + ((TW * wv + t) * CT + x) * 1024 + lane * 16) = dg[t][x];
            if (i > 0) keep(a.gm, L::S, u, NP, NS);
            DeltaParts<C, NP> f[CS][CT];
            frags(L::OG, f);
#pragma unroll
            for (int t = 0; t < TW; ++t)
#pragma unroll
                for (int x = 0; x < CT; ++x) dg[t][x] = zero;
            into(dg, f, [&](int r, int p) { return slice + r * L::SROW + p * 16; }, 0);
#pragma unroll
            for (int x = 0; x < CT; ++x) du[x] = zero;
#pragma unroll
            for (int sl = 0; sl < CS; ++sl)
                if (used(sl))
#pragma unroll
                    for (int x = 0; x < CT; ++x) {
                        DeltaParts<C, 1> y;
                        y.p[0] = frag1(L::O, sl, x, 1);
                        du[x] = delta_mma(M[T2][sl], y, du[x]);
                    }
            mn = moved(mn, ahead, then, dtri);
            load_tri(mn, M[T2]);
            ahead = then;
            lds_barrier();
#pragma unroll
            for (int x = 0; x < CT; ++x) *reinterpret_cast<f32x4*>(smem + L::DU + (wv * CT + x) * 1024 + lane * 16) = du[x];
            lds_barrier();
            if (i > 0) keep(a.ym, L::V, u, 1, CS);
        };
        in_turn(round);
        // the last round, in which they are at the last chunk: nothing is left to bring (what it computes again nobody takes)
        if (NC & 1) round(std::integral_constant<int, 1>{}, NC, first + NC * step);
        else round(std::integral_constant<int, 0>{}, NC, first + NC * step);
        }
        if (!walk_again(most_out > END)) return;
    }
}

template <typename T, int D, int CT, int MODE>
static hipError_t launch(const DeltaArgs& a, hipStream_t stream) {
    typedef ScanLds<T, D, CT, MODE> L;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&delta_scan_kernel<T, D, CT, MODE>), hipFuncAttributeMaxDynamicSharedMemorySize, L::BYTES);
    if (attr != hipSuccess) return attr;
    const int nseg = MODE == DELTA_O ? a.nseg : MODE == DELTA_PART ? a.nseg - 1 : 1, parts = D / 16 / CT * (MODE == DELTA_PART ? 2 : 1);
    delta_scan_kernel<T, D, CT, MODE><<<dim3(xcd_deal_grid(parts, a.nseq * a.V * nseg)), dim3(512), L::BYTES, stream>>>(a);
    return hipGetLastError();
}
// 32 columns to a workgroup where those of 16 do not all find a CU: each chunk's K, Q and matrices then serve twice as many.  4096 tokens, d = 128, 16 against 32 columns, uncut, all kernels, us:
// 32 heads 125 and 153 (training forward 159, 181), 40 heads 210 and 160 (276, 209), 64 heads 254 and 196 (351, 260).
template <typename T, int D, int MODE>
static hipError_t launch_ct(const DeltaArgs& a, hipStream_t stream) {
    if constexpr (sizeof(T) == 2 || D == 64)      // (fp32 at d = 128: 32 columns do not fit the registers; 16 spill 62, of the training pair 74 and 48)
        if (MODE == DELTA_PART || a.nseg > 1 || (long long)a.nseq * a.V * (D / 16) > 256) return launch<T, D, 2, MODE>(a, stream);
    return launch<T, D, 1, MODE>(a, stream);
}
template <int D, int MODE>
static hipError_t launch_type(const DeltaArgs& a, int is_bf16, hipStream_t stream) {
    return is_bf16 ? launch_ct<bf16_t, D, MODE>(a, stream) : launch_ct<float, D, MODE>(a, stream);
}
template <int D> static hipError_t launch_mode(const DeltaArgs& a, int is_bf16, int mode, hipStream_t stream) {
    if (mode == DELTA_KEEP) return launch_type<D, DELTA_KEEP>(a, is_bf16, stream);
    if (mode == DELTA_BACK) return launch_type<D, DELTA_BACK>(a, is_bf16, stream);
    if (a.nseg > 1)
        if (const hipError_t e = launch_type<D, DELTA_PART>(a, is_bf16, stream)) return e;
    return launch_type<D, DELTA_O>(a, is_bf16, stream);
}
hipError_t launch_delta_scan(const DeltaArgs& a, int d, int is_bf16, int mode, hipStream_t stream) {
    return d == 64 ? launch_mode<64>(a, is_bf16, mode, stream) : launch_mode<128>(a, is_bf16, mode, stream);
}

// Segments of sequences whose longest has `chunks`.  Heads are dealt to 8 XCDs of 32 CUs, a workgroup takes a CU: both launches are to fit at once.  Beyond the root of 0.6 times the chunks
// the joining of states costs more than shorter segments gain, and two segments gain nothing.  Times in us, both launches and the matrices of the chunks, d = 128, one sequence:
//   8 heads of 16384 tokens   1 segment 358, 2: 442, 3: 312, 4: 251, 5 (taken): 215, 6 (does not fit): 250       16 heads of 8192   1: 199, 2: 245, 3 (taken): 182, 4: 199
//   4 heads of 4096           1: 95, 3: 93, 4: 81, 6 (taken): 69, 12: 81                                          1 head of 2560     1: 64, 4 (taken): 59, 6: 54, 12: 61
// fp32 at d = 128, whose workgroups have 16 columns: 8 heads of 16384 3 segments (taken) 612, 5 (more than fit) 735; 4 heads of 4096 111, 127.
int delta_segments(long long units, int d, int is_bf16, long long chunks) {
    int n = 1;
    if (chunks < DELTA_CUT) return 1;
    const int cols = !is_bf16 && d == 128 ? 16 : 32;      // of a workgroup (launch_ct)
    while ((units * n + 7) / 8 * (2 * d / cols) <= 32 && (units * (n + 1) + 7) / 8 * (d / cols) <= 32 && 10ll * (n + 1) * (n + 1) <= 6 * chunks) ++n;
    return n >= 3 ? n : 1;
}

}  // namespace path
