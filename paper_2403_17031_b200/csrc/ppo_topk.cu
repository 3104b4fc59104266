// Log-probs of given tokens with entropy, log-sum-exp and the k most likely alternatives of every row, in one pass
// over the logits (ppo_logprob_topk), and the gradient on all of those back to the logits (ppo_logprob_topk_bwd).
//
// Forward. The statistics are those of step 1: sums of 2^(y - ref) and 2^(y - ref) (y - ref) with y = logit log2(e) /
// temperature, relative to a reference per warp. Beside them every thread keeps the maximum of the elements it streams
// (packs tid, tid + 256, ...), for each half of them (a "segment") on its own. (Short rows: 128 threads with one segment each.)
// Selection then works on those:
//   the k-th largest of the threads' maxima is a threshold t with at least k elements >= t, so nothing below t is
//   among the k best; only segments whose maximum reaches t hold candidates. Every segment's maximum comes with its pack and
//   the largest value outside that pack, so most of these segments (about k of 512) need that one pack re-read, by the thread
//   that streamed it, and only those with a second pack that reaches t are searched whole, by half a warp: for 997 rows of
//   50277 fp32, k = 64, one segment in 150. (Searching all of them is sector traffic of more than the row: 85 us instead of
//   39 for these rows. One segment per thread: 51 us, k = 20 the same 37; four: 39, but 91 instead of 81 us for 3392 bf16
//   rows.) Candidates are ranked by counting against each other on the 64-bit key (value, ~index), which is unique: ties go to
//   the lowest index and the order in which candidates arrive does not matter.
// A slice whose candidates overflow the list (rows of equal values, fewer than k unbanned tokens) is selected by
// radix passes over it instead.
// Few rows: a cluster of CL blocks shares a row; each selects the k best of its slice, and block 0 ranks what is
// in their lists and merges the sums, through distributed shared memory.
// Bound: the read of the logits (V * size bytes per row; without alternatives 3392 x 50304 bf16 57 us = 6.0 TB/s), and behind it
// the selection, which the other rows of an SM have to cover: k = 5: 64 us, k = 20: 68 us, half the rows masked, k = 5: 38 us =
// 4.5 TB/s (1.4 rounds of blocks); one row, k = 20: 7.7 us.
#include <cooperative_groups.h>

#include "ppo_rows.cuh"

namespace ppo {
namespace topk {

namespace cg = cooperative_groups;

constexpr int kSharedK = 32;      // from here on the blocks of a cluster share a threshold
constexpr int kMaxIds = 128;       // largest k and largest number of given tokens

struct Args {
    const void *logits;
    int V;
    int64_t row_stride;
    const int32_t *tokens;
    int n;
    const uint8_t *mask;
    float c;
    int k;
    float *logprob, *entropy, *lse;
    int32_t *top_ids;
    float *top_logprob;
    int *status;
};

// What a thread knows of a segment: the maximum, the largest value outside the pack that holds it, that pack.
struct Segment {
    float top, second;
    int pack;
    __device__ __forceinline__ void init()
    {
        top = second = -INFINITY;
        pack = 0x7fffffff;
    }
    __device__ __forceinline__ void add(float xmax, int i)
    {
        second = fmaxf(second, fminf(xmax, top));
        pack = xmax > top ? i : pack;
        top = fmaxf(top, xmax);
    }
};

// of a block of TH threads, one of CL that share a row
template <int CL, int TH>
struct Smem {
    static constexpr int kThreads = TH;
    static constexpr int kParts = TH == 256 ? 2 : 1;         // segments of a thread
    static constexpr int kCap = CL == 1 ? 512 : 1280;        // candidates: with several blocks also their merged lists
    unsigned long long cand[kCap];
    unsigned long long best[kMaxIds];    // the slice's best, sorted
    uint32_t seg_key[256];               // maxima of the threads' elements as ordered keys; the fallback's histogram
    Segment seg[kParts][kThreads];
    float red[96];
    SoftmaxState st;
    uint32_t threshold, second_threshold;
    int n_cand, n_best, bin, need;
};

// whole numbers that order like the values (-0 equals +0); 0 is below every value
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return (b >> 31) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float((u >> 31) ? (u & 0x7fffffffu) : ~u); }
__device__ __forceinline__ unsigned long long make_key(uint32_t u, int j)
{
    return ((unsigned long long)u << 32) | (uint32_t)~(uint32_t)j;
}

// One pack into the sums (clamped at kNegBig, so a -inf logit adds exact zeros) and into the segment.
template <typename T>
__device__ __forceinline__ void accumulate(const uint4 &v, int i, float c, float nm, FixedAcc &a, Segment &seg)
{
    float x[Pack<T>::N], xmax;
    Pack<T>::unpack(v, x, xmax);
    seg.add(xmax, i);
    const float2 cc = make_float2(c, c), nn = make_float2(nm, nm);
    float2 s = make_float2(a.s0, a.s1), u = make_float2(a.u0, a.u1);
#pragma unroll
    for (int q = 0; q < Pack<T>::N; q += 2) {
        const float2 t = __ffma2_rn(make_float2(x[q], x[q + 1]), cc, nn);
        const float2 e = make_float2(ex2(t.x), ex2(t.y));
        s = __fadd2_rn(s, e);
        u = __ffma2_rn(e, t, u);
    }
    a.s0 = s.x; a.s1 = s.y;
    a.u0 = u.x; a.u1 = u.y;
}

__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, off));
    return v;
}

// What block `rank` of CL handles of a row: elements [e0, e1), of which packs [p0, p1) of the 16-byte aligned body
// (body element i of the row is head + i) and at most 2 (N - 1) loose elements at the row's ends.
struct Slice {
    int head, p0, p1, e0, e1, loose;
};

template <typename T>
__device__ __forceinline__ Slice slice_of(const T *src, int V, int rank, int CL)
{
    constexpr int N = Pack<T>::N;
    Slice s;
    s.head = min(V, (int)(((16u - (reinterpret_cast<uintptr_t>(src) & 15u)) & 15u) / sizeof(T)));
    const int nvec = (V - s.head) / N;
    const int per = (nvec + CL - 1) / CL;
    s.p0 = min(nvec, rank * per);
    s.p1 = min(nvec, s.p0 + per);
    s.e0 = rank == 0 ? 0 : s.head + s.p0 * N;
    s.e1 = rank == CL - 1 ? V : s.head + s.p1 * N;
    s.loose = s.e1 - s.e0 - (s.p1 - s.p0) * N;
    return s;
}

// element index of the slice's loose element number t, or -1
template <typename T>
__device__ __forceinline__ int loose_element(const Slice &s, int t)
{
    constexpr int N = Pack<T>::N;
    const int lead = (s.e0 == 0) ? s.head : 0;
    if (t < lead) return t;
    const int j = s.head + s.p1 * N + (t - lead);
    return j < s.e1 ? j : -1;
}

// The k best of elements [e0, e1) into sm.cand (unsorted, k of them), for any values: radix passes find the k-th
// largest value, then all larger ones and the first of the equal ones (in index order) are taken.
template <typename T, typename S>
__device__ __noinline__ void select_by_radix(const T *src, int e0, int e1, int k, S &sm)
{
    constexpr int kThreads = S::kThreads, kWarps = kThreads / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint32_t prefix = 0;
    int need = k;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kThreads) sm.seg_key[i] = 0;
        __syncthreads();
        for (int j0 = e0; j0 < e1; j0 += kThreads) {
            const int j = j0 + tid;
            uint32_t u = 0;
            bool active = j < e1;
            if (active) {
                u = ordered(Pack<T>::load1(src + j));
                active = shift == 24 || (u >> (shift + 8)) == prefix;
            }
            const uint32_t votes = __ballot_sync(0xffffffffu, active);
            if (active) {
                const uint32_t bin = (u >> shift) & 255u, peers = __match_any_sync(votes, bin);
                if (lane == __ffs(peers) - 1) atomicAdd(&sm.seg_key[bin], (uint32_t)__popc(peers));
            }
        }
        __syncthreads();
        if (tid == 0) {
            int bin = 255, left = need;
            for (; bin > 0 && (int)sm.seg_key[bin] < left; --bin) left -= (int)sm.seg_key[bin];
            sm.bin = bin;
            sm.need = left;
        }
        __syncthreads();
        prefix = (prefix << 8) | (uint32_t)sm.bin;
        need = sm.need;
        __syncthreads();
    }
    const int greater = k - need;                        // strictly above the k-th value
    if (tid == 0) sm.n_cand = 0;
    __syncthreads();
    int taken = 0;
    for (int j0 = e0; j0 < e1; j0 += kThreads) {
        const int j = j0 + tid;
        const uint32_t u = j < e1 ? ordered(Pack<T>::load1(src + j)) : 0;
        if (u > prefix) sm.cand[atomicAdd(&sm.n_cand, 1)] = make_key(u, j);
        if (taken < need) {                              // the same in every thread
            const bool tie = j < e1 && u == prefix;
            const uint32_t votes = __ballot_sync(0xffffffffu, tie);
            if (lane == 0) sm.seg_key[warp] = (uint32_t)__popc(votes);
            __syncthreads();
            int before = taken, total = 0;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                if (w < warp) before += (int)sm.seg_key[w];
                total += (int)sm.seg_key[w];
            }
            before += __popc(votes & ((1u << lane) - 1u));
            if (tie && before < need) sm.cand[greater + before] = make_key(u, j);
            taken += total;
            __syncthreads();
        }
    }
    __syncthreads();
    if (tid == 0) sm.n_cand = k;
    __syncthreads();
}

// Warp 0: a threshold that at least k and at most a few more of the threads' maxima reach.
template <typename S>
__device__ __forceinline__ void choose_threshold(int k, const S &sm, uint32_t &threshold)
{
    constexpr int Q = S::kThreads / 32;
    const int lane = threadIdx.x & 31;
    uint32_t key[Q], top = 0, low = 0xffffffffu;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        key[q] = sm.seg_key[q * 32 + lane];
        top = max(top, key[q]);
        low = min(low, key[q]);
    }
    uint32_t lo = __reduce_min_sync(0xffffffffu, low), hi = __reduce_max_sync(0xffffffffu, top);
    // invariant: count(>= lo) >= k (there are more threads than k); count(> hi) = 0
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo + 1) / 2;
        int cnt = 0;
#pragma unroll
        for (int q = 0; q < Q; ++q) cnt += key[q] >= mid;
        cnt = (int)__reduce_add_sync(0xffffffffu, (unsigned)cnt);
        if (cnt >= k) {
            lo = mid;
            if (cnt <= k + (k >> 3) + 3) break;
        } else {
            hi = mid - 1;
        }
    }
    // maxima are clamped at kNegBig: at that level everything is a candidate
    if (lane == 0) threshold = lo <= ordered(0.99f * kNegBig) ? 0u : lo;
}

// the elements of a pack that reach the threshold into the list of candidates
template <typename T, typename S>
__device__ __forceinline__ void take_candidates(const uint4 &v, int at, int head, float thr, S &sm)
{
    constexpr int N = Pack<T>::N;
    float x[N];
    Pack<T>::unpack_raw(v, x);
    float top = x[0];
#pragma unroll
    for (int e = 1; e < N; ++e) top = fmaxf(top, x[e]);
    if (!(top >= thr)) return;
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (x[e] >= thr) {
            const int c = atomicAdd(&sm.n_cand, 1);
            if (c < S::kCap) sm.cand[c] = make_key(ordered(x[e]), head + at * N + e);
        }
}

// the `want` best of n candidates into sm.best, sorted
template <typename S>
__device__ __forceinline__ void rank_candidates(int n, int want, S &sm)
{
    for (int i = threadIdx.x; i < n; i += S::kThreads) {
        const unsigned long long key = sm.cand[i];
        int rank = 0;
        int j = 0;
        for (; j + 4 <= n; j += 4) {
            rank += sm.cand[j] > key;
            rank += sm.cand[j + 1] > key;
            rank += sm.cand[j + 2] > key;
            rank += sm.cand[j + 3] > key;
        }
        for (; j < n; ++j) rank += sm.cand[j] > key;
        if (rank < want) sm.best[rank] = key;
    }
}

// The slice's best elements into sm.best, sorted: those that reach the threshold, k at most. Loose elements are in sm.cand
// already. `span`: packs of a segment.
template <typename T, typename S>
__device__ __forceinline__ void select_best(const T *src, const Slice &sl, int span, int k, uint32_t threshold, S &sm)
{
    constexpr int kThreads = S::kThreads, kParts = S::kParts;
    const int tid = threadIdx.x, lane = tid & 31;
    const int want = min(k, sl.e1 - sl.e0);
    const float thr = threshold == 0u ? -INFINITY : unordered(threshold);
    const uint4 *body = reinterpret_cast<const uint4 *>(src + sl.head);
    // a thread re-reads the one pack of its segments with candidates in no other
    uint4 v[kParts];
    int at[kParts];
    bool whole[kParts];
#pragma unroll
    for (int s = 0; s < kParts; ++s) {
        const Segment g = sm.seg[s][tid];
        whole[s] = g.second >= thr;
        at[s] = g.top >= thr && !whole[s] ? g.pack : sl.p1;
        if (at[s] < sl.p1) v[s] = body[at[s]];
    }
#pragma unroll
    for (int s = 0; s < kParts; ++s)
        if (at[s] < sl.p1) take_candidates<T>(v[s], at[s], sl.head, thr, sm);
    // the others are searched by half a warp each
#pragma unroll
    for (int s = 0; s < kParts; ++s) {
        uint32_t todo = __ballot_sync(0xffffffffu, whole[s]);
        while (todo) {
            const int l0 = __ffs(todo) - 1;
            todo &= todo - 1;
            const int l1 = __ffs(todo) - 1;                 // -1: none
            todo &= todo - 1;
            const int l = lane < 16 ? l0 : l1;
            const int first = l < 0 ? sl.p1 : sl.p0 + (tid & ~31) + l + s * span * kThreads;
            for (int j = lane & 15; j < span; j += 16) {
                const int i = first + j * kThreads;
                if (i < sl.p1) take_candidates<T>(body[i], i, sl.head, thr, sm);
            }
        }
    }
    __syncthreads();
    if (sm.n_cand > S::kCap) {
        __syncthreads();
        select_by_radix(src, sl.e0, sl.e1, want, sm);
    }
    const int n = sm.n_cand;
    rank_candidates(n, want, sm);
    if (tid == 0) sm.n_best = min(n, want);
    __syncthreads();
}

// (a block to a row: 8 blocks of 256 threads to an SM, 32 registers a thread, hide the selection of some behind the streams
// of the others better than four loads in flight per thread and 4 blocks do: 38 against 41 us for 3392 bf16 rows, half of them
// masked, 39 against 46 for 997 fp32; what the stream does not need is therefore loaded behind it. Clusters: four blocks have to
// fit, two let some of 37 clusters of 8 wait: 36 rows 7.5 us instead of 12)
template <typename T, int CL, int TH>
__global__ void __launch_bounds__(TH, CL == 1 ? 2048 / TH : 4)
topk_kernel(const Args a)
{
    constexpr int kThreads = TH, kWarps = TH / 32, kParts = Smem<CL, TH>::kParts;
    __shared__ Smem<CL, TH> sm;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x / CL;
    const int rank = blockIdx.x % CL;
    if (a.mask && !a.mask[row]) {
        if (rank == 0) {
            if (tid < a.n) a.logprob[row * a.n + tid] = 0.f;
            if (tid < a.k) {
                a.top_ids[row * a.k + tid] = -1;
                a.top_logprob[row * a.k + tid] = 0.f;
            }
            if (tid == 0) {
                if (a.entropy) a.entropy[row] = 0.f;
                if (a.lse) a.lse[row] = 0.f;
            }
        }
        return;
    }
    const T *src = reinterpret_cast<const T *>(a.logits) + row * a.row_stride;
    const Slice sl = slice_of(src, a.V, rank, CL);
    const uint4 *body = reinterpret_cast<const uint4 *>(src + sl.head);
    // Sums are taken relative to the maximum of the warp's first loads (about a thousand elements, all of them when the
    // row is split eightfold): near the row's own maximum, so that the entropy, a difference of two numbers that grow
    // with the distance, keeps its digits.
    FixedAcc acc;
    acc.init();
    Segment seg;
    seg.init();
    constexpr int U = CL == 1 ? 2 : 4;
    // packs of a segment: a thread's share in kParts parts, whole rounds of loads
    const int per_thread = (sl.p1 - sl.p0 + kThreads - 1) / kThreads, span = ((per_thread + kParts - 1) / kParts + U - 1) / U * U;
    int part = 0;
    const int lane = tid & 31, warp = tid >> 5;
    uint4 v[U];
    float first_max = kNegBig;
    int i = sl.p0 + tid;
#pragma unroll
    for (int q = 0; q < U; ++q)
        if (i + q * kThreads < sl.p1) v[q] = ld_stream(body + i + q * kThreads);
#pragma unroll
    for (int q = 0; q < U; ++q)
        if (i + q * kThreads < sl.p1) {
            float x[Pack<T>::N], xmax;
            Pack<T>::unpack(v[q], x, xmax);
            first_max = fmaxf(first_max, xmax);
        }
    const float w_max = warp_max(first_max);
    const float m_warp = safe_reference(w_max, a.c), nm = -m_warp;
    // (a warp whose first loads hold no logit with weight has no reference: its sums are marked as overflown)
    if (w_max <= kNoWeight) acc.s0 = INFINITY;
#pragma unroll
    for (int q = 0; q < U; ++q)
        if (i + q * kThreads < sl.p1) accumulate<T>(v[q], i + q * kThreads, a.c, nm, acc, seg);
    i += U * kThreads;
    int next = sl.p0 + tid + span * kThreads;
    const auto next_part = [&] {
        sm.seg[part++][tid] = seg;
        seg.init();
        next += span * kThreads;
    };
    while (true) {
        for (const int end = min(next, sl.p1 - (U - 1) * kThreads); i < end; i += U * kThreads) {
#pragma unroll
            for (int q = 0; q < U; ++q) v[q] = ld_stream(body + i + q * kThreads);
#pragma unroll
            for (int q = 0; q < U; ++q) accumulate<T>(v[q], i + q * kThreads, a.c, nm, acc, seg);
        }
        if (i != next) break;
        next_part();
    }
#pragma unroll
    for (int q = 0; q < U - 1; ++q)
        if (i + q * kThreads < sl.p1) v[q] = ld_stream(body + i + q * kThreads);
#pragma unroll
    for (int q = 0; q < U - 1; ++q)
        if (i + q * kThreads < sl.p1) accumulate<T>(v[q], i + q * kThreads, a.c, nm, acc, seg);
    float x_tok = 0.f;
    bool tok_ok = true;
    if (rank == 0 && tid < a.n) {
        const int tok = a.tokens[row * a.n + tid];
        tok_ok = (unsigned)tok < (unsigned)a.V;
        if (tok_ok) x_tok = Pack<T>::load1(src + tok);
    }
    const int loose = tid < 2 * (Pack<T>::N - 1) ? loose_element<T>(sl, tid) : -1;
    const float x_loose = loose >= 0 ? Pack<float>::clampf(Pack<T>::load1(src + loose)) : kNegBig;
    SoftmaxState st;
    st.m = m_warp;
    st.s = acc.s0 + acc.s1;
    st.u = acc.u0 + acc.u1;
    if (loose >= 0) st.add(fmaf(x_loose, a.c, nm));
    if (!(st.s < kSumLimit) || !(fabsf(st.u) < kSumLimit)) {   // too far above (or NaN / +inf): again with a moving reference
        init_online(st);
        for (i = sl.p0 + tid; i < sl.p1; i += kThreads) accumulate_online<T>(body[i], a.c, st);
        if (loose >= 0) {
            const float y = x_loose * a.c;
            if (y > st.m) st.rebase(y);
            st.add(exponent_of(x_loose, a.c, -st.m));
        }
    }
    // within the warp plain sums unless a lane moved its reference, then the eight warps' states by the general rule
    if (__any_sync(0xffffffffu, st.m != m_warp)) {
        st = warp_merge(st);
    } else {
        st.s = warp_sum_f(st.s);
        st.u = warp_sum_f(st.u);
    }
    if (lane == 0) { sm.red[warp] = st.m; sm.red[32 + warp] = st.s; sm.red[64 + warp] = st.u; }
    if (a.k > 0) {
        float top = seg.top;
        while (part < kParts) next_part();                 // (those behind the current one are empty)
#pragma unroll
        for (int s = 0; s < kParts; ++s) top = fmaxf(top, sm.seg[s][tid].top);
        sm.seg_key[tid] = sl.p0 + tid < sl.p1 ? ordered(top) : 0u;
        if (loose >= 0) sm.cand[tid] = make_key(ordered(Pack<T>::load1(src + loose)), loose);   // (they come first)
        if (tid == 0) sm.n_cand = sl.loose;
    }
    __syncthreads();
    // With several blocks and k large, each finds a threshold that k / CL of its threads reach; the lowest of them has at least
    // k elements of the row above it, and the lists stay short (one row of 50304, k = 128: 9.4 us, with lists of k from each block
    // 40; from k = 32 on it is worth the exchange: k = 20, 120 rows: 10.6 us with it, 10.0 without).
    const bool shared = CL > 1 && a.k >= kSharedK;
    if (warp == 0 && a.k > 0) choose_threshold(shared ? (a.k + CL - 1) / CL : a.k, sm, sm.threshold);
    if (warp == 1) {
        st.init();
        if (lane < kWarps) { st.m = sm.red[lane]; st.s = sm.red[32 + lane]; st.u = sm.red[64 + lane]; }
        st = warp_merge(st);
        if (lane == 0) sm.st = st;
    }
    __syncthreads();
    st = sm.st;
    uint32_t threshold = a.k > 0 ? sm.threshold : 0u;
    if (shared) {
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        const uint32_t of_lane = *cluster.map_shared_rank(&sm.threshold, lane % CL);
        threshold = __reduce_min_sync(0xffffffffu, of_lane);
        const int alive = __popc(__ballot_sync(0xffffffffu, of_lane != 0u)) / (32 / CL);
        if (threshold == 0u && alive > 0) {                // blocks of banned tokens: the others find k among themselves
            if (warp == 0) choose_threshold((a.k + alive - 1) / alive, sm, sm.second_threshold);
            cluster.sync();
            const uint32_t second = *cluster.map_shared_rank(&sm.second_threshold, lane % CL);
            threshold = __reduce_min_sync(0xffffffffu, of_lane != 0u ? second : 0xffffffffu);
        }
    }
    if (a.k > 0) {
        // (false for NaN; a slice without weight, s = 0, is selected from)
        if (st.s < 1.0e37f) {
            select_best(src, sl, span, a.k, threshold, sm);
        } else {
            if (tid == 0) sm.n_best = 0;
            __syncthreads();
        }
    }
    if (CL > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        if (rank == 0) {
            st.init();
            int len = 0;
            if (lane < CL) {
                st = *cluster.map_shared_rank(&sm.st, lane);
                if (a.k > 0) len = *cluster.map_shared_rank(&sm.n_best, lane);
            }
            st = warp_merge(st);
            if (a.k > 0) {
                // warp r fetches the list of block r, to behind those of the blocks before it
                int end = len;
#pragma unroll
                for (int off = 1; off < CL; off *= 2) {
                    const int before = __shfl_up_sync(0xffffffffu, end, off);
                    if (lane >= off) end += before;
                }
                const int n = __shfl_sync(0xffffffffu, end, CL - 1);
                const int to = __shfl_sync(0xffffffffu, end - len, warp), mine = __shfl_sync(0xffffffffu, len, warp);
                if (warp < CL) {
                    const unsigned long long *from = cluster.map_shared_rank(&sm.best[0], warp);
                    for (int q = lane; q < mine; q += 32) sm.cand[to + q] = from[q];
                }
                __syncthreads();
                rank_candidates(n, a.k, sm);
                __syncthreads();
            }
        }
        cluster.sync();
        if (rank != 0) return;
    }
    // (beyond 2^30 the rounding error of the reference, ref - x*c, leaves fp32's range as an exponent: any sum may come out)
    const bool good = st.s > 0.f && st.s < 1.0e37f && fabsf(st.m) < 1073741824.f;
    const float nan = __uint_as_float(0x7fffffffu);
    const float l2s = log2f(st.s);
    // In base-2 units the log-sum-exp is m + log2 s with m possibly in the thousands. Log-probs subtract it in fp64
    // (a few values per row), so they are as accurate as their own size; lse itself is rounded once.
    const double ln2 = 0.69314718055994530942, lse2 = (double)st.m + (double)l2s, c = (double)a.c;
    const float lse = good ? (float)(lse2 * ln2) : nan;
    if (tid < a.n) {
        a.logprob[row * a.n + tid] = good && tok_ok ? (float)(((double)x_tok * c - lse2) * ln2) : nan;
        if (!tok_ok && a.status) atomicOr(a.status, PPO_DEV_BAD_TOKEN);
    }
    if (tid < a.k) {
        const unsigned long long key = sm.best[tid];
        a.top_ids[row * a.k + tid] = good ? (int)~(uint32_t)key : -1;
        a.top_logprob[row * a.k + tid] = good ? (float)(((double)unordered((uint32_t)(key >> 32)) * c - lse2) * ln2) : nan;
    }
    if (tid == 0) {
        if (a.entropy) a.entropy[row] = good ? (float)(((double)l2s - (double)st.u / (double)st.s) * ln2) : nan;
        if (a.lse) a.lse[row] = lse;
        if (!good && a.status) atomicOr(a.status, PPO_DEV_BAD_ROW);
    }
}

template <typename T, int CL, int TH>
static int launch(const Args &a, int64_t rows, cudaStream_t s)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * CL));
    cfg.blockDim = dim3(TH);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CL;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CL > 1 ? 1 : 0;
    PPO_RETURN_IF_CUDA(cudaLaunchKernelEx(&cfg, topk_kernel<T, CL, TH>, a));
    return PPO_OK;
}

template <typename T>
static int launch_any(const Args &a, int64_t rows, cudaStream_t s)
{
    // few rows: split each over a cluster while there are SMs to fill and every thread still streams a pack or more
    const int64_t packs = a.V / Pack<T>::N;
    if (rows * 8 <= 2 * 148 && packs >= 8 * 256) return launch<T, 8, 256>(a, rows, s);
    if (rows * 4 <= 2 * 148 && packs >= 4 * 256) return launch<T, 4, 256>(a, rows, s);
    // (pairs for more rows if they are long: 250 rows of 50277 fp32 15 us instead of 20; shorter ones lose: 50304 bf16 12
    // instead of 11)
    if (rows * 2 <= (packs >= 8192 ? 4 : 2) * 148 && packs >= 2 * 256) return launch<T, 2, 256>(a, rows, s);
    // Short rows, enough of them to fill the SMs, few alternatives: half the threads and twice the blocks on an SM, so that more
    // selections hide each other. bf16, 128 against 256 threads: 3392 x 4096, k = 20: 17 / 23 us, 3392 x 16384: 29 / 36 us; 200 x
    // 16384: 8.6 / 7.5 us; 1000 x 16384, k = 64: 18.7 / 17.2 us; 997 x 50277 fp32 (longer rows), k = 20: 46 / 37 us.
    if (packs <= 2048 && rows >= 4 * 148 && a.k <= 32) return launch<T, 1, 128>(a, rows, s);
    return launch<T, 1, 256>(a, rows, s);
}

// ---------------------------------------------------------------- backward
// With p_j = exp(z_j - lse), G the sum of all given gradients and h the gradient on the entropy H:
//     dlogits_j = ( p_j (dlse - G - h (ln p_j + H)) + sum of the gradients given for token j ) / temperature
// One read and one write of the row; the statistics come from the forward call. A block handles a chunk of a row: it
// writes the dense part, then the elements that are given tokens once more with their gradients added (all in fp32,
// rounded once; a token given several times is summed in the order given, by the first of its places).
// Bound: bytes (read + write of the logits' size): 3392 x 50304 bf16, half the rows masked, 86 us = 6.0 TB/s.
constexpr int kBwdThreads = 256, kBwdWarps = kBwdThreads / 32;

struct BwdArgs {
    const void *logits;
    void *dlogits;
    int V, chunks, packs_per_chunk;
    int64_t ls, ds;
    const int32_t *tokens, *top_ids;
    const float *dlogprob, *dtop;
    int n, k;
    const float *lse, *entropy, *dentropy, *dlse;
    const uint8_t *mask;
    float c_hi, c_lo, inv_tau;      // log2(e) / temperature as a sum of two floats
    int *status;
};

struct RowTerm {
    float c_hi, c_lo, o_hi, o_lo, a0, a1;
    // log2 p, accurate to a few ulps of itself however large z and lse are
    __device__ __forceinline__ float log2p(float x) const
    {
        const float t = fmaf(x, c_hi, -o_hi);
        return t < -200.f ? -200.f : t + fmaf(x, c_lo, -o_lo);   // p is 0 there, -inf included (a NaN stays one)
    }
    __device__ __forceinline__ float grad(float x) const
    {
        const float t = log2p(x);
        return ex2(t) * fmaf(a1, t, a0);
    }
};

template <typename T>
__global__ void __launch_bounds__(kBwdThreads)
topk_bwd_kernel(const BwdArgs a)
{
    constexpr int N = Pack<T>::N, U = 2;
    __shared__ float red[kBwdWarps];
    __shared__ int ids[2 * kMaxIds];
    __shared__ float gs[2 * kMaxIds];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t row = blockIdx.x / a.chunks;
    const int chunk = blockIdx.x % a.chunks;
    const T *src = reinterpret_cast<const T *>(a.logits) + row * a.ls;
    T *dst = reinterpret_cast<T *>(a.dlogits) + row * a.ds;
    // packs are aligned in dlogits; where the logits sit at another offset they are read element by element
    const int head = min(a.V, (int)(((16u - (reinterpret_cast<uintptr_t>(dst) & 15u)) & 15u) / sizeof(T)));
    const int nvec = (a.V - head) / N;
    const int p0 = chunk * a.packs_per_chunk, p1 = min(nvec, p0 + a.packs_per_chunk);
    const bool first = chunk == 0, last = chunk == a.chunks - 1;
    const int e0 = first ? 0 : head + p0 * N, e1 = last ? a.V : head + p1 * N;
    uint4 *out = reinterpret_cast<uint4 *>(dst + head);
    // loose elements: before the first pack of the row and behind its last
    int loose = -1;
    if (first && tid < head) loose = tid;
    if (last && tid >= 32 && tid - 32 < a.V - head - nvec * N) loose = head + nvec * N + (tid - 32);
    if (a.mask && !a.mask[row]) {
        const uint4 z = make_uint4(0u, 0u, 0u, 0u);
        for (int i = p0 + tid; i < p1; i += kBwdThreads) st_stream(out + i, z);
        if (loose >= 0) Pack<T>::store1(dst + loose, 0.f);
        return;
    }
    const bool vec_in = ((reinterpret_cast<uintptr_t>(src + head) & 15u) == 0);
    const uint4 *in = reinterpret_cast<const uint4 *>(src + head);
    uint4 v[U];
    const int i0 = p0 + tid;
    if (vec_in) {
#pragma unroll
        for (int q = 0; q < U; ++q)
            if (i0 + q * kBwdThreads < p1) v[q] = ld_stream(in + i0 + q * kBwdThreads);
    }
    // the given tokens and the sum of their gradients
    const int total = a.n + a.k;
    int id = 0;
    float g = 0.f;
    if (tid < total) {
        const bool top = tid >= a.n;
        const int64_t at = top ? row * a.k + (tid - a.n) : row * a.n + tid;
        id = top ? a.top_ids[at] : a.tokens[at];
        g = top ? a.dtop[at] : a.dlogprob[at];
        ids[tid] = id;
        gs[tid] = g;
    }
    const float wsum = warp_sum_f(g);
    if (lane == 0) red[warp] = wsum;
    const int bad = __syncthreads_or((unsigned)id >= (unsigned)a.V);
    float G = 0.f;
#pragma unroll
    for (int w = 0; w < kBwdWarps; ++w) G += red[w];
    RowTerm r;
    {
        const float lse = a.lse[row], h = a.dentropy ? a.dentropy[row] : 0.f, H = a.dentropy ? a.entropy[row] : 0.f;
        const double off = (double)lse * 1.4426950408889634074;
        r.c_hi = a.c_hi;
        r.c_lo = a.c_lo;
        r.o_hi = (float)off;
        r.o_lo = (float)(off - (double)r.o_hi);
        r.a0 = ((a.dlse ? a.dlse[row] : 0.f) - G - h * H) * a.inv_tau;
        r.a1 = -h * kLn2 * a.inv_tau;
        if (bad) r.a0 = __uint_as_float(0x7fffffffu);
    }
    if (bad && chunk == 0 && tid == 0 && a.status) atomicOr(a.status, PPO_DEV_BAD_TOKEN);
    for (int i = i0; i < p1; i += U * kBwdThreads) {
        if (vec_in && i != i0) {
#pragma unroll
            for (int q = 0; q < U; ++q)
                if (i + q * kBwdThreads < p1) v[q] = ld_stream(in + i + q * kBwdThreads);
        }
#pragma unroll
        for (int q = 0; q < U; ++q) {
            const int p = i + q * kBwdThreads;
            if (p >= p1) continue;
            float x[N];
            if (vec_in) {
                Pack<T>::unpack_raw(v[q], x);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) x[e] = Pack<T>::load1(src + head + p * N + e);
            }
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = r.grad(x[e]);
            st_stream(out + p, Pack<T>::pack(x));
        }
    }
    if (loose >= 0) Pack<T>::store1(dst + loose, r.grad(Pack<T>::load1(src + loose)));
    __syncthreads();
    if (tid < total && !bad && id >= e0 && id < e1) {
        float sum = 0.f;
        bool owner = true;
        for (int j = 0; j < total; ++j)
            if (ids[j] == id) {
                owner = owner && j >= tid;
                sum += gs[j];
            }
        if (owner) Pack<T>::store1(dst + id, fmaf(sum, a.inv_tau, r.grad(Pack<T>::load1(src + id))));
    }
}

template <typename T>
static int launch_bwd(BwdArgs a, int64_t rows, cudaStream_t s)
{
    const int nvec = a.V / Pack<T>::N;
    // a block's share: 2048 packs (32 KB in, 32 KB out) once there are blocks for every place on the SMs, so that its reads
    // of the row's tokens and gradients weigh little (1024: 95 us instead of 86 for 3392 bf16 rows); else 1024, for more
    // blocks (4.7 us instead of 5.6 for 53 rows)
    a.packs_per_chunk = (rows * (nvec / (8 * kBwdThreads) + 1) >= 8 * 148 ? 8 : 4) * kBwdThreads;
    a.chunks = nvec > 0 ? (nvec + a.packs_per_chunk - 1) / a.packs_per_chunk : 1;
    const int64_t blocks = rows * a.chunks;
    if (blocks >= ((int64_t)1 << 31)) return PPO_ERR_SHAPE;
    topk_bwd_kernel<T><<<(unsigned)blocks, kBwdThreads, 0, s>>>(a);
    return launch_status();
}

}   // namespace topk
}   // namespace ppo

using namespace ppo;

extern "C" int ppo_logprob_topk(const void *logits, int dtype, int64_t rows, int64_t V, int64_t row_stride,
                                const int32_t *tokens, int32_t n, const uint8_t *mask, float temperature, int32_t k,
                                float *logprob, float *entropy, float *lse, int32_t *top_ids, float *top_logprob,
                                void *workspace, void *stream)
{
    if (dtype != PPO_F32 && dtype != PPO_BF16) return PPO_ERR_DTYPE;
    if (rows < 0 || rows >= ((int64_t)1 << 31) || V <= 0 || V >= ((int64_t)1 << 31) - 512 || row_stride < V || n < 0 ||
        n > topk::kMaxIds || k < 0 || k > topk::kMaxIds || k > V)
        return PPO_ERR_SHAPE;
    if (!(temperature > 0.f) || !finite_f(temperature)) return PPO_ERR_PARAM;
    if (rows == 0) return PPO_OK;
    if (!logits || (n > 0 && (!tokens || !logprob)) || (k > 0 && (!top_ids || !top_logprob))) return PPO_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(logits) % (dtype == PPO_F32 ? 4 : 2)) return PPO_ERR_ALIGN;
    topk::Args a = {};
    a.logits = logits;
    a.V = (int)V;
    a.row_stride = row_stride;
    a.tokens = tokens;
    a.n = n;
    a.mask = mask;
    a.c = (float)(1.4426950408889634074 / (double)temperature);
    a.k = k;
    a.logprob = logprob;
    a.entropy = entropy;
    a.lse = lse;
    a.top_ids = top_ids;
    a.top_logprob = top_logprob;
    a.status = workspace ? &ws_header(workspace)->status : nullptr;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    return dtype == PPO_F32 ? topk::launch_any<float>(a, rows, s) : topk::launch_any<__nv_bfloat16>(a, rows, s);
}

extern "C" int ppo_logprob_topk_bwd(const void *logits, int dtype, int64_t rows, int64_t V, int64_t row_stride,
                                    const int32_t *tokens, int32_t n, const float *dlogprob, const int32_t *top_ids,
                                    int32_t k, const float *dtop_logprob, const float *lse, const float *entropy,
                                    const float *dentropy, const float *dlse, const uint8_t *mask, float temperature,
                                    void *dlogits, int64_t dlogits_stride, void *workspace, void *stream)
{
    if (dtype != PPO_F32 && dtype != PPO_BF16) return PPO_ERR_DTYPE;
    if (rows < 0 || rows >= ((int64_t)1 << 31) || V <= 0 || V >= ((int64_t)1 << 31) - 512 || row_stride < V ||
        dlogits_stride < V || n < 0 || n > topk::kMaxIds || k < 0 || k > topk::kMaxIds)
        return PPO_ERR_SHAPE;
    if (!(temperature > 0.f) || !finite_f(temperature)) return PPO_ERR_PARAM;
    if (rows == 0) return PPO_OK;
    if (!logits || !dlogits || !lse || (n > 0 && (!tokens || !dlogprob)) || (k > 0 && (!top_ids || !dtop_logprob)) ||
        (dentropy && !entropy))
        return PPO_ERR_NULL;
    if (logits == dlogits) return PPO_ERR_PARAM;
    const size_t es = dtype == PPO_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(logits) % es || reinterpret_cast<uintptr_t>(dlogits) % es) return PPO_ERR_ALIGN;
    topk::BwdArgs a = {};
    a.logits = logits;
    a.dlogits = dlogits;
    a.V = (int)V;
    a.ls = row_stride;
    a.ds = dlogits_stride;
    a.tokens = tokens;
    a.n = n;
    a.dlogprob = dlogprob;
    a.top_ids = top_ids;
    a.k = k;
    a.dtop = dtop_logprob;
    a.lse = lse;
    a.entropy = entropy;
    a.dentropy = dentropy;
    a.dlse = dlse;
    a.mask = mask;
    const double c = 1.4426950408889634074 / (double)temperature;
    a.c_hi = (float)c;
    a.c_lo = (float)(c - (double)a.c_hi);
    a.inv_tau = 1.0f / temperature;
    a.status = workspace ? &ws_header(workspace)->status : nullptr;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    return dtype == PPO_F32 ? topk::launch_bwd<float>(a, rows, s) : topk::launch_bwd<__nv_bfloat16>(a, rows, s);
}
