// Page tables made to fit the requests' lengths: pages behind the tokens that stay go back to the stack of free ones, new tokens get pages off its top, both in the
// order of the table; then the offsets of the packed new tokens and the cache slot of each.  Integers throughout, no atomics: the same call gives the same tables.
//
// Bound by latency: launches that depend on each other, each a chain of a few reads.  What a sequence adds to sums over the ones before it is read again by every
// sequence (a wave's 64 lanes at a time), which is cheaper than a launch of its own for the sums.
#include "plan_decl.h"

namespace path {

namespace {
__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
    for (int i = 1; i < 64; i *= 2) x += __shfl_xor(x, i);
    return x;
}
__device__ __forceinline__ long long wave_sum(long long x) {
#pragma unroll
    for (int i = 1; i < 64; i *= 2) x += __shfl_xor(x, i);
    return x;
}
__device__ __forceinline__ int held(int x) { return x < 0 ? 0 : x; }

// sum of x[0 .. n), not below 0 each, by a wave, N reads of a lane together
template <int N> __device__ __forceinline__ long long sum_before(const int* x, int n, int lane) {
    long long y = 0;
    for (int i0 = 0; i0 < n; i0 += 64 * N) {
        int v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0;
            if (i0 + 64 * i < n) v[i] = x[i0 + 64 * i + lane < n ? i0 + 64 * i + lane : n - 1];
        }
#pragma unroll
        for (int i = 0; i < N; ++i) y += i0 + 64 * i + lane < n ? held(v[i]) : 0;
    }
    return wave_sum(y);
}

struct Row { int* entries; int have, want; long long start, end; };      // of a sequence: its entries, pages with cached tokens, pages wanted, first new token and the one behind the last
__device__ __forceinline__ Row row_of(const PlanArgs& a, int s, long long start) {
    Row r;
    r.entries = a.table + (size_t)s * a.per_seq;
    long long end = start + held(a.fresh[s]);
    r.start = start < a.T ? start : a.T;
    r.end = end < a.T ? end : a.T;
    const long long n = held(a.cached[s]), page = 1LL << a.shift, have = (n + page - 1) >> a.shift, want = (n + r.end - r.start + page - 1) >> a.shift;
    r.want = (int)(want < a.per_seq ? want : a.per_seq);
    r.have = (int)(have < a.per_seq ? have : a.per_seq);
    return r;
}
__device__ __forceinline__ bool page_ok(const PlanArgs& a, int e) { return e >= 0 && e < a.num_pages; }
__device__ __forceinline__ int free_at_first(const PlanArgs& a) { const int c = a.scratch[0]; return c < 0 ? 0 : c > a.num_pages ? a.num_pages : c; }

// Entries j0 .. of a row, 64 apart per lane, N of a lane requested together.  One after the other, 2048 of them took 10 us, the latency of 32 reads, eight at a time 6; in the kernel of one workgroup, whose
// rows are short, the longer code costs 1.5 us instead.
template <int N> __device__ __forceinline__ void read_ahead(const PlanArgs& a, const Row& r, int j0, int lane, int (&e)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int j = j0 + 64 * i + lane;
        e[i] = -1;
        if (j0 + 64 * i < a.per_seq) e[i] = r.entries[j < a.per_seq ? j : a.per_seq - 1];
    }
}

// What each sequence gives back and wants.
template <int N> __device__ void plan_count(const PlanArgs& a, int s, int lane) {
    const Row r = row_of(a, s, sum_before<N>(a.fresh, s, lane));
    int back = 0, need = 0;
    for (int j0 = (r.have < r.want ? r.have : r.want) / 64 * 64; j0 < a.per_seq; j0 += N * 64) {
        int e[N];
        read_ahead(a, r, j0, lane, e);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int j = j0 + 64 * i + lane;
            const bool ok = page_ok(a, e[i]);
            back += ok && j >= r.want && j < a.per_seq;
            need += !ok && j >= r.have && j < r.want;
        }
    }
    back = wave_sum(back);
    need = wave_sum(need);
    if (lane == 0) {
        a.cu[s] = (int)r.start;
        if (s == a.nseq - 1) a.cu[a.nseq] = (int)r.end;
        a.scratch[1 + s] = back;
        a.scratch[1 + a.nseq + s] = need;
        if (s == 0) a.scratch[0] = a.count[0];
    }
}
// Pages go back.  (Entries that are no page, and what finds no room on the stack, go nowhere.)
template <int N> __device__ void plan_back(const PlanArgs& a, int s, int lane) {
    const Row r = row_of(a, s, a.cu[s]);      // (held already: the same pages)
    long long at = free_at_first(a) + sum_before<N>(a.scratch + 1, s, lane);
    for (int j0 = r.want / 64 * 64; j0 < a.per_seq; j0 += N * 64) {
        int e[N];
        read_ahead(a, r, j0, lane, e);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int j = j0 + 64 * i + lane;
            const bool mine = j >= r.want && j < a.per_seq, page = mine && page_ok(a, e[i]);
            const unsigned long long ok = __ballot(page);
            if (page) {
                const long long place = at + __popcll(ok & ((1ull << lane) - 1));
                if (place < a.num_pages) a.free_pages[place] = e[i];
            }
            if (mine && e[i] != -1) r.entries[j] = -1;
            at += __popcll(ok);
        }
    }
}
// Pages are taken.
template <int N> __device__ void plan_take(const PlanArgs& a, int s, int lane) {
    const Row r = row_of(a, s, a.cu[s]);
    const long long back = sum_before<N>(a.scratch + 1, a.nseq, lane), before = sum_before<N>(a.scratch + 1 + a.nseq, s, lane);
    const long long all = free_at_first(a) + back, top = all < a.num_pages ? all : a.num_pages;
    const int need = a.scratch[1 + a.nseq + s];
    long long at = top - 1 - before;
    int missing = 0;
    if (need > 0)
        for (int j0 = r.have / 64 * 64; j0 < r.want; j0 += 64) {
            const int j = j0 + lane;
            const bool mine = j >= r.have && j < r.want && !page_ok(a, r.entries[j]);
            const unsigned long long who = __ballot(mine);
            if (mine) {
                const long long place = at - __popcll(who & ((1ull << lane) - 1));
                r.entries[j] = place >= 0 ? a.free_pages[place] : -1;
                missing += place < 0;
            }
            at -= __popcll(who);
        }
    missing = wave_sum(missing);
    if (lane == 0) {
        a.missing[s] = missing;
        if (s == a.nseq - 1) a.count[0] = (int)(top - before - need > 0 ? top - before - need : 0);
    }
}
// Slots of tokens t0, t0 + step, .. below t1, by a workgroup's threads.
__device__ void plan_map(const PlanArgs& a, long long t0, long long t1, int step) {
    for (long long t = t0; t < t1; t += step) {
        int lo = 0, hi = a.nseq;      // the sequence: how many end at or before t
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (a.cu[mid + 1] <= t) lo = mid + 1; else hi = mid;
        }
        long long slot = -1;
        if (lo < a.nseq) {
            const long long pos = held(a.cached[lo]) + (t - a.cu[lo]), j = pos >> a.shift;
            if (j < a.per_seq) {
                const int e = a.table[(size_t)lo * a.per_seq + j];
                if (page_ok(a, e)) slot = ((long long)e << a.shift) + (pos & ((1LL << a.shift) - 1));
            }
        }
        a.slots[t] = slot;
    }
}
}  // namespace

__global__ __launch_bounds__(1024) void plan_small_kernel(PlanArgs a) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    for (int s = wv; s < a.nseq; s += 16) plan_count<1>(a, s, lane);
    __syncthreads();
    for (int s = wv; s < a.nseq; s += 16) plan_back<1>(a, s, lane);
    __syncthreads();
    for (int s = wv; s < a.nseq; s += 16) plan_take<1>(a, s, lane);
    __syncthreads();
    plan_map(a, threadIdx.x, a.T, 1024);
}
template <int PHASE> __global__ __launch_bounds__(256) void plan_rows_kernel(PlanArgs a) {
    const int lane = threadIdx.x & 63, s = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (s >= a.nseq) return;
    if (PHASE == 0) plan_count<8>(a, s, lane);
    if (PHASE == 1) plan_back<8>(a, s, lane);
    if (PHASE == 2) plan_take<8>(a, s, lane);
}
__global__ __launch_bounds__(256) void plan_map_kernel(PlanArgs a) {
    const long long t = (long long)blockIdx.x * 256 + threadIdx.x;
    plan_map(a, t, t < a.T ? t + 1 : t, 1);
}

hipError_t launch_plan(const PlanArgs& a, hipStream_t stream) {
    // One workgroup has 16 waves, a row each: two rows to a wave are level with four launches (32 rows of 256 entries 10.7 us against 33 rows' 11.3 and three more starts, 16 of 64 6.3; 128 of 64 31 against
    // 13, 512 of 16 148 against 15).
    if ((long long)a.nseq * a.per_seq <= 8192 && a.nseq <= 32 && a.T <= 4096) {
        plan_small_kernel<<<dim3(1), dim3(1024), 0, stream>>>(a);
        return hipGetLastError();
    }
    const dim3 rows((a.nseq + 3) / 4), threads(256);
    plan_rows_kernel<0><<<rows, threads, 0, stream>>>(a);
    plan_rows_kernel<1><<<rows, threads, 0, stream>>>(a);
    plan_rows_kernel<2><<<rows, threads, 0, stream>>>(a);
    if (a.T > 0) plan_map_kernel<<<dim3((unsigned)(((long long)a.T + 255) / 256)), threads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace path
