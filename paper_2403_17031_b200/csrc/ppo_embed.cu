// The input embedding: rows of a table, scaled (ppo_embed), and the gradient of the table (ppo_embed_bwd).
//
//     out[i, :] = scale * E[tokens[i], :]                       dE[v, :] = scale * sum over i with tokens[i] = v of dY[i, :]
//
// Both move bytes and do next to no arithmetic. The forward call reads each row once from memory (rows that occur again
// come from L2) and writes N rows. The gradient reads N rows and writes V, most of them zeros when N is small.
//
// Gradient: the positions are sorted by token (stable), so that the rows of one token follow one another. The sorted list
// is cut into chunks of equal length, whatever the tokens: text has a few tokens that make up a large share of it, and a
// block per token would leave them to a few blocks. A run of one token inside a chunk is summed in registers and
// written once; a run that crosses chunks leaves a partial sum per chunk, and those are added in the order of the chunks.
// Every sum is fp32 in ascending order of the positions, without atomics: results do not depend on timing. Rows of tokens
// that do not occur are zero-filled by other blocks of the same launch.
#include "ppo_common.cuh"

namespace ppo {
namespace embed {

constexpr int kThreads = 256;

// ---------------------------------------------------------------- loads and stores of VEC elements as fp32
template <typename T, int VEC> struct Pack;
template <> struct Pack<float, 1> {
    float v[1];
    __device__ __forceinline__ void load(const float *p) { v[0] = __ldg(p); }
    __device__ __forceinline__ void load_last(const float *p) { v[0] = __ldcs(p); }
    __device__ __forceinline__ static void store(float *p, const float *x) { __stcs(p, x[0]); }
};
template <> struct Pack<__nv_bfloat16, 1> {
    float v[1];
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { v[0] = __bfloat162float(*p); }
    __device__ __forceinline__ void load_last(const __nv_bfloat16 *p) { v[0] = __bfloat162float(*p); }
    __device__ __forceinline__ static void store(__nv_bfloat16 *p, const float *x) { *p = __float2bfloat16_rn(x[0]); }
};
template <> struct Pack<float, 8> {
    float v[8];
    __device__ __forceinline__ void set(const float4 &a, const float4 &b)
    {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
    __device__ __forceinline__ void load(const float *p)
    {
        set(__ldg(reinterpret_cast<const float4 *>(p)), __ldg(reinterpret_cast<const float4 *>(p) + 1));
    }
    __device__ __forceinline__ void load_last(const float *p)
    {
        set(__ldcs(reinterpret_cast<const float4 *>(p)), __ldcs(reinterpret_cast<const float4 *>(p) + 1));
    }
    __device__ __forceinline__ static void store(float *p, const float *x)
    {
        __stcs(reinterpret_cast<float4 *>(p), make_float4(x[0], x[1], x[2], x[3]));
        __stcs(reinterpret_cast<float4 *>(p) + 1, make_float4(x[4], x[5], x[6], x[7]));
    }
};
template <> struct Pack<__nv_bfloat16, 8> {
    float v[8];
    __device__ __forceinline__ void set(const uint4 &a)
    {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = __uint_as_float(w[j] << 16);
            v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { set(__ldg(reinterpret_cast<const uint4 *>(p))); }
    __device__ __forceinline__ void load_last(const __nv_bfloat16 *p) { set(__ldcs(reinterpret_cast<const uint4 *>(p))); }
    __device__ __forceinline__ static void store(__nv_bfloat16 *p, const float *x)
    {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]);
            w[j] = *reinterpret_cast<const uint32_t *>(&h);
        }
        __stcs(reinterpret_cast<uint4 *>(p), make_uint4(w[0], w[1], w[2], w[3]));
    }
};

// A thread's columns of a row: Q packs of VEC neighbours, packs `lanes` apart so that a warp's accesses are contiguous.
// VEC 8 where all rows are 16-byte aligned, else single elements, four of them in flight.
template <int VEC> __host__ __device__ constexpr int packs_per_thread() { return VEC == 8 ? 1 : 4; }

static bool aligned_rows(const void *p, int64_t pitch, int dtype)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && pitch % (dtype == PPO_F32 ? 4 : 8) == 0;
}

// ---------------------------------------------------------------- forward
struct FwdArgs {
    const void *table;
    const int32_t *tokens;
    void *out;
    int64_t N, V, lde, ldo;
    int K;
    float scale;
    int *status;
};

// One block per ROWS rows; the rows' loads are issued before the first store.
template <typename TI, typename TO, int VEC, int ROWS>
__global__ void __launch_bounds__(kThreads)
lookup_kernel(const FwdArgs a)
{
    const int64_t i0 = (int64_t)blockIdx.x * ROWS;
    const TI *row[ROWS];
    float scale[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        row[r] = reinterpret_cast<const TI *>(a.table);
        scale[r] = a.scale;
        if (i0 + r < a.N) {
            const int t = a.tokens[i0 + r];
            const bool ok = t >= 0 && t < a.V;
            if (ok) row[r] += (int64_t)t * a.lde;
            else scale[r] = __int_as_float(0x7fc00000);
            if (!ok && threadIdx.x == 0 && a.status) atomicOr(a.status, PPO_DEV_BAD_TOKEN);
        }
    }
    TO *out = reinterpret_cast<TO *>(a.out) + i0 * a.ldo;
    for (int k = threadIdx.x * VEC; k < a.K; k += kThreads * VEC) {
        Pack<TI, VEC> p[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) p[r].load(row[r] + k);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) p[r].v[e] *= scale[r];
            if (i0 + r < a.N) Pack<TO, VEC>::store(out + r * a.ldo + k, p[r].v);
        }
    }
}

template <typename TI, typename TO>
static int launch_lookup(const FwdArgs &a, bool vec, cudaStream_t s)
{
    // four rows per block once they fill the SMs
    const bool many = a.N >= 4 * 8 * 148;
    const unsigned grid = (unsigned)(many ? (a.N + 3) / 4 : a.N);
    if (vec && many) lookup_kernel<TI, TO, 8, 4><<<grid, kThreads, 0, s>>>(a);
    else if (vec) lookup_kernel<TI, TO, 8, 1><<<grid, kThreads, 0, s>>>(a);
    else if (many) lookup_kernel<TI, TO, 1, 4><<<grid, kThreads, 0, s>>>(a);
    else lookup_kernel<TI, TO, 1, 1><<<grid, kThreads, 0, s>>>(a);
    return launch_status();
}

// ---------------------------------------------------------------- sorting the positions by token
// Keys are token ids; a position that counts for no row (padding id, id outside [0, V)) has the key V and comes last.
struct SortArgs {
    const int32_t *tokens;
    int64_t V;
    int N, padding_id;
    int32_t *key, *pos;            // sorted
    uint8_t *present;              // [V], cleared before; nullable
    int *status;
};

__device__ __forceinline__ int key_of(const SortArgs &a, int i)
{
    const int t = a.tokens[i];
    return t < 0 || t >= a.V || t == a.padding_id ? (int)a.V : t;
}

__device__ __forceinline__ void note_token(const SortArgs &a, int i, int key)
{
    if (key < a.V) {
        if (a.present) a.present[key] = 1;
    } else if (a.status) {
        const int t = a.tokens[i];
        if (t < 0 || t >= a.V) atomicOr(a.status, PPO_DEV_BAD_TOKEN);
    }
}

// Few positions: each one's place is the number of positions before it, counted. A warp counts for four positions.
constexpr int kRankPer = 4, kRankMax = 8192;
__global__ void __launch_bounds__(kThreads)
rank_kernel(const SortArgs a)
{
    const int lane = threadIdx.x & 31;
    const int i0 = (blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * kRankPer;
    if (i0 >= a.N) return;
    int key[kRankPer], n[kRankPer];
#pragma unroll
    for (int r = 0; r < kRankPer; ++r) {
        key[r] = i0 + r < a.N ? key_of(a, i0 + r) : 0;
        n[r] = 0;
    }
#pragma unroll 4
    for (int j = lane; j < a.N; j += 32) {
        const int k = key_of(a, j);
#pragma unroll
        for (int r = 0; r < kRankPer; ++r) n[r] += k < key[r] || (k == key[r] && j < i0 + r);
    }
#pragma unroll
    for (int r = 0; r < kRankPer; ++r) {
        n[r] = __reduce_add_sync(0xffffffffu, n[r]);
        if (lane == r && i0 + r < a.N) {
            a.key[n[r]] = key[r];
            a.pos[n[r]] = i0 + r;
            note_token(a, i0 + r, key[r]);
        }
    }
}

// Many positions: least significant digit first, 8 bits a pass, each pass stable: digits counted per tile, the counts
// summed in digit order, the tile's entries moved. A warp owns 512 neighbouring entries of a tile.
constexpr int kTile = 4096, kDigits = 256, kWarps = kThreads / 32, kPerWarp = kTile / kWarps;

struct PassArgs {
    SortArgs s;
    const int32_t *key_in, *pos_in;      // null in the first pass
    int32_t *key_out, *pos_out;
    int32_t *counts;                     // [kDigits][tiles]
    int tiles, shift, last;
};

__device__ __forceinline__ void load_entry(const PassArgs &a, int i, int &key, int &pos)
{
    key = a.key_in ? a.key_in[i] : key_of(a.s, i);
    pos = a.pos_in ? a.pos_in[i] : i;
}

__global__ void __launch_bounds__(kThreads)
count_kernel(const PassArgs a)
{
    __shared__ int n[kDigits];
    n[threadIdx.x] = 0;
    __syncthreads();
    const int i0 = blockIdx.x * kTile;
#pragma unroll 4
    for (int j = threadIdx.x; j < kTile; j += kThreads) {
        if (i0 + j < a.s.N) {
            int key, pos;
            load_entry(a, i0 + j, key, pos);
            atomicAdd(&n[(key >> a.shift) & (kDigits - 1)], 1);
        }
    }
    __syncthreads();
    a.counts[(size_t)threadIdx.x * a.tiles + blockIdx.x] = n[threadIdx.x];
}

// exclusive sum over `n` counts, in place; one block
constexpr int kScanThreads = 1024;
__global__ void __launch_bounds__(kScanThreads)
scan_kernel(int32_t *__restrict__ counts, int n)
{
    __shared__ int warp_sum[32];
    __shared__ int carry;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) carry = 0;
    __syncthreads();
    for (int base = 0; base < n; base += kScanThreads * 8) {
        const int i = base + threadIdx.x * 8;
        int v[8], sum = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = i + e < n ? counts[i + e] : 0;
            sum += v[e];
        }
        int incl = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += o;
        }
        if (lane == 31) warp_sum[warp] = incl;
        __syncthreads();
        int before = carry;
        for (int w = 0; w < warp; ++w) before += warp_sum[w];
        int run = before + incl - sum;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (i + e < n) counts[i + e] = run;
            run += v[e];
        }
        __syncthreads();
        if (threadIdx.x == kScanThreads - 1) carry = run;
        __syncthreads();
    }
}

__global__ void __launch_bounds__(kThreads)
scatter_kernel(const PassArgs a)
{
    __shared__ int at[kWarps][kDigits];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int j = threadIdx.x; j < kWarps * kDigits; j += kThreads) (&at[0][0])[j] = 0;
    __syncthreads();
    const int i0 = blockIdx.x * kTile + warp * kPerWarp;
    for (int j = lane; j < kPerWarp; j += 32) {
        if (i0 + j < a.s.N) {
            int key, pos;
            load_entry(a, i0 + j, key, pos);
            atomicAdd(&at[warp][(key >> a.shift) & (kDigits - 1)], 1);
        }
    }
    __syncthreads();
    {   // the warps' first places of each digit
        int run = a.counts[(size_t)threadIdx.x * a.tiles + blockIdx.x];
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const int n = at[w][threadIdx.x];
            at[w][threadIdx.x] = run;
            run += n;
        }
    }
    __syncthreads();
    for (int j = lane; j < kPerWarp; j += 32) {
        const bool in = i0 + j < a.s.N;
        int key = 0, pos = 0;
        if (in) load_entry(a, i0 + j, key, pos);
        const int digit = in ? (key >> a.shift) & (kDigits - 1) : kDigits;
        const unsigned same = __match_any_sync(0xffffffffu, digit);
        const int before = __popc(same & ((1u << lane) - 1));
        int to = 0;
        if (in) to = at[warp][digit] + before;
        __syncwarp();
        if (in && before == 0) at[warp][digit] += __popc(same);
        __syncwarp();
        if (in) {
            a.key_out[to] = key;
            a.pos_out[to] = pos;
            if (a.last) note_token(a.s, pos, key);
        }
    }
}

// ---------------------------------------------------------------- sums
struct BwdArgs {
    const void *dY;
    const int32_t *key, *pos;       // sorted
    const uint8_t *present;
    void *dE;
    float *part;                    // [chunks][2][K]: a run that comes from the chunk before; one that goes on in the next
    int64_t V, ldy, lde;
    int N, K, chunk, chunks, accumulate;
    float scale;
    int lanes, groups, slabs;       // threads per chunk and slab, chunks per block (lanes * groups = kThreads)
    int chunk_blocks, fill_rows;    // blocks that sum; rows per block of the others
};

template <typename TO, int VEC>
__device__ __forceinline__ void write_row(const BwdArgs &a, int64_t v, int k, float *x)
{
    TO *to = reinterpret_cast<TO *>(a.dE) + v * a.lde + k;
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] *= a.scale;
    if (a.accumulate) {
        Pack<TO, VEC> old;
        old.load_last(to);
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[e] += old.v[e];
    }
    Pack<TO, VEC>::store(to, x);
}

template <typename TI, typename TO, int VEC>
__global__ void __launch_bounds__(kThreads)
sum_kernel(const BwdArgs a)
{
    constexpr int Q = packs_per_thread<VEC>(), U = 8 / Q;      // rows in flight
    if ((int)blockIdx.x >= a.chunk_blocks) {
        // zero rows
        const int64_t v0 = (int64_t)(blockIdx.x - a.chunk_blocks) * a.fill_rows;
        float zero[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) zero[e] = 0.f;
        for (int64_t v = v0; v < v0 + a.fill_rows && v < a.V; ++v) {
            if (a.present[v]) continue;
            TO *to = reinterpret_cast<TO *>(a.dE) + v * a.lde;
            for (int k = threadIdx.x * VEC; k < a.K; k += kThreads * VEC) Pack<TO, VEC>::store(to + k, zero);
        }
        return;
    }
    const int lane = threadIdx.x % a.lanes, group = threadIdx.x / a.lanes;
    const int slab = blockIdx.x % a.slabs, c = (blockIdx.x / a.slabs) * a.groups + group;
    if (c >= a.chunks) return;
    int k[Q];
    bool in[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        k[q] = ((slab * Q + q) * a.lanes + lane) * VEC;
        in[q] = k[q] < a.K;
    }
    const int e0 = c * a.chunk, e1 = min(e0 + a.chunk, a.N);
    const TI *dY = reinterpret_cast<const TI *>(a.dY);
    float acc[Q][VEC];
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[q][e] = 0.f;
    int cur = a.key[e0];
    bool from_before = e0 > 0 && a.key[e0 - 1] == cur;
    const auto flush = [&](bool goes_on) {
        if (cur >= a.V) return;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            if (!in[q]) continue;
            if (from_before || goes_on) {
                float *to = a.part + ((size_t)c * 2 + (from_before ? 0 : 1)) * a.K + k[q];
#pragma unroll
                for (int e = 0; e < VEC; ++e) to[e] = acc[q][e];
            } else {
                write_row<TO, VEC>(a, cur, k[q], acc[q]);
            }
        }
    };
    for (int e = e0; e < e1 && cur < a.V; e += U) {
        Pack<TI, VEC> p[U][Q];
        int key[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            key[u] = e + u < e1 ? a.key[e + u] : -1;
            const bool real = key[u] >= 0 && key[u] < a.V;
            const TI *row = dY + (real ? (int64_t)a.pos[e + u] : 0) * a.ldy;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                if (real && in[q]) p[u][q].load_last(row + k[q]);
                else
#pragma unroll
                    for (int x = 0; x < VEC; ++x) p[u][q].v[x] = 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (key[u] >= 0 && key[u] != cur) {
                flush(false);
                cur = key[u];
                from_before = false;
#pragma unroll
                for (int q = 0; q < Q; ++q)
#pragma unroll
                    for (int x = 0; x < VEC; ++x) acc[q][x] = 0.f;
            }
#pragma unroll
            for (int q = 0; q < Q; ++q)
#pragma unroll
                for (int x = 0; x < VEC; ++x) acc[q][x] += p[u][q].v[x];
        }
    }
    flush(e1 < a.N && a.key[e1] == cur);
}

// The runs that cross chunks: the block of the chunk in which such a run begins adds the partial sums up.
template <typename TO>
__global__ void __launch_bounds__(kThreads)
join_kernel(const BwdArgs a)
{
    const int c = blockIdx.x / a.slabs, k0 = (blockIdx.x % a.slabs) * kThreads + threadIdx.x;
    const int e0 = c * a.chunk, e1 = e0 + a.chunk;              // (the last chunk has no block)
    const int t = a.key[e1 - 1];
    if (t >= a.V || a.key[e1] != t) return;                     // no run goes on
    if (e0 > 0 && a.key[e0 - 1] == t) return;                   // it began in an earlier chunk
    int lo = c + 1, hi = a.chunks - 1;                          // last chunk that begins with t
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.key[(size_t)mid * a.chunk] == t) lo = mid;
        else hi = mid - 1;
    }
    if (k0 >= a.K) return;
    float sum = a.part[((size_t)c * 2 + 1) * a.K + k0];
#pragma unroll 8
    for (int i = c + 1; i <= lo; ++i) sum += a.part[(size_t)i * 2 * a.K + k0];
    write_row<TO, 1>(a, t, k0, &sum);
}

// ---------------------------------------------------------------- host side
struct Plan {
    int chunk, chunks, lanes, groups, slabs, tiles, passes;
    size_t key, pos, key2, pos2, counts, present, part, bytes;
};

static Plan plan_of(int64_t N, int64_t K, int64_t V, bool vec)
{
    Plan p;
    const int64_t packs = vec ? (K + 7) / 8 : (K + 3) / 4;      // threads for a row
    p.lanes = 8;
    while (p.lanes < kThreads && p.lanes < packs) p.lanes *= 2;
    p.groups = kThreads / p.lanes;
    p.slabs = (int)((packs + p.lanes - 1) / p.lanes);
    p.chunk = N > 65536 ? 128 : 32;
    p.chunks = (int)((N + p.chunk - 1) / p.chunk);
    p.tiles = N <= kRankMax ? 0 : (int)((N + kTile - 1) / kTile);
    p.passes = 0;
    if (p.tiles) {
        int bits = 1;
        while (bits < 32 && (V >> bits)) ++bits;
        p.passes = (bits + 7) / 8;
    }
    size_t at = 0;
    const auto take = [&](size_t n) {
        const size_t here = at;
        at += align256(n);
        return here;
    };
    p.key = take((size_t)N * 4);
    p.pos = take((size_t)N * 4);
    p.key2 = take(p.tiles ? (size_t)N * 4 : 0);
    p.pos2 = take(p.tiles ? (size_t)N * 4 : 0);
    p.counts = take((size_t)p.tiles * kDigits * 4);
    p.present = take((size_t)V);
    p.part = take((size_t)p.chunks * 2 * (size_t)K * 4);
    p.bytes = at;
    return p;
}

static int launch_sort(const SortArgs &sa, const Plan &p, unsigned char *scratch, cudaStream_t s)
{
    if (!p.tiles) {
        const int per_block = kThreads / 32 * kRankPer;
        rank_kernel<<<(sa.N + per_block - 1) / per_block, kThreads, 0, s>>>(sa);
        return launch_status();
    }
    PassArgs a = {};
    a.s = sa;
    a.tiles = p.tiles;
    a.counts = reinterpret_cast<int32_t *>(scratch + p.counts);
    int32_t *key[2] = {sa.key, reinterpret_cast<int32_t *>(scratch + p.key2)};
    int32_t *pos[2] = {sa.pos, reinterpret_cast<int32_t *>(scratch + p.pos2)};
    int to = (p.passes & 1) ^ 1;                                // the last pass writes the first pair
    for (int pass = 0; pass < p.passes; ++pass, to ^= 1) {
        a.key_out = key[to];
        a.pos_out = pos[to];
        a.shift = pass * 8;
        a.last = pass == p.passes - 1;
        count_kernel<<<p.tiles, kThreads, 0, s>>>(a);
        int rc = launch_status();
        if (rc) return rc;
        scan_kernel<<<1, kScanThreads, 0, s>>>(a.counts, p.tiles * kDigits);
        rc = launch_status();
        if (rc) return rc;
        scatter_kernel<<<p.tiles, kThreads, 0, s>>>(a);
        rc = launch_status();
        if (rc) return rc;
        a.key_in = a.key_out;
        a.pos_in = a.pos_out;
    }
    return PPO_OK;
}

template <typename TI, typename TO>
static int launch_sums(const BwdArgs &a, bool vec, cudaStream_t s)
{
    const int64_t fill = a.accumulate ? 0 : (a.V + a.fill_rows - 1) / a.fill_rows;
    const unsigned grid = (unsigned)(a.chunk_blocks + fill);
    if (vec) sum_kernel<TI, TO, 8><<<grid, kThreads, 0, s>>>(a);
    else sum_kernel<TI, TO, 1><<<grid, kThreads, 0, s>>>(a);
    int rc = launch_status();
    if (rc || a.chunks < 2) return rc;
    BwdArgs j = a;
    j.slabs = (a.K + kThreads - 1) / kThreads;
    join_kernel<TO><<<(unsigned)((a.chunks - 1) * j.slabs), kThreads, 0, s>>>(j);
    return launch_status();
}

static bool dtype_ok(int d) { return d == PPO_F32 || d == PPO_BF16; }
static size_t size_of(int d) { return d == PPO_F32 ? 4 : 2; }
constexpr int64_t kLimit = ((int64_t)1 << 31) - 8192;

}   // namespace embed
}   // namespace ppo

using namespace ppo;

extern "C" int ppo_embed(const void *table, int dtype, int64_t V, int64_t K, int64_t lde, const int32_t *tokens, int64_t N,
                         float scale, void *out, int out_dtype, int64_t ldo, void *workspace, void *stream)
{
    using namespace embed;
    if (!dtype_ok(dtype) || !dtype_ok(out_dtype)) return PPO_ERR_DTYPE;
    if (N < 0 || K <= 0 || V <= 0 || N >= kLimit || K >= kLimit || V >= kLimit || lde < K || ldo < K) return PPO_ERR_SHAPE;
    if (!finite_f(scale)) return PPO_ERR_PARAM;
    if (N == 0) return PPO_OK;
    if (!table || !tokens || !out) return PPO_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(table) % size_of(dtype) || reinterpret_cast<uintptr_t>(out) % size_of(out_dtype) ||
        reinterpret_cast<uintptr_t>(tokens) % 4)
        return PPO_ERR_ALIGN;
    FwdArgs a = {};
    a.table = table; a.tokens = tokens; a.out = out;
    a.N = N; a.V = V; a.K = (int)K; a.lde = lde; a.ldo = ldo; a.scale = scale;
    a.status = workspace ? &ws_header(workspace)->status : nullptr;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const bool vec = K % 8 == 0 && aligned_rows(table, lde, dtype) && aligned_rows(out, ldo, out_dtype);
    if (dtype == PPO_F32)
        return out_dtype == PPO_F32 ? launch_lookup<float, float>(a, vec, s) : launch_lookup<float, __nv_bfloat16>(a, vec, s);
    return out_dtype == PPO_F32 ? launch_lookup<__nv_bfloat16, float>(a, vec, s) : launch_lookup<__nv_bfloat16, __nv_bfloat16>(a, vec, s);
}

extern "C" size_t ppo_embed_bwd_scratch_bytes(int64_t N, int64_t K, int64_t V)
{
    using namespace embed;
    if (N <= 0 || K <= 0 || V <= 0 || N >= kLimit || K >= kLimit || V >= kLimit) return 0;
    return plan_of(N, K, V, false).bytes;
}

extern "C" int ppo_embed_bwd(const void *dY, int dtype, int64_t N, int64_t K, int64_t ldy, const int32_t *tokens, int64_t V,
                             float scale, int32_t padding_id, void *dE, int out_dtype, int64_t lde, int accumulate,
                             void *workspace, void *scratch, void *stream)
{
    using namespace embed;
    if (!dtype_ok(dtype) || !dtype_ok(out_dtype)) return PPO_ERR_DTYPE;
    if (N < 0 || K <= 0 || V <= 0 || N >= kLimit || K >= kLimit || V >= kLimit || ldy < K || lde < K) return PPO_ERR_SHAPE;
    if (!finite_f(scale)) return PPO_ERR_PARAM;
    if (!dE) return PPO_ERR_NULL;
    if (N > 0 && (!dY || !tokens || !scratch)) return PPO_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(dY) % size_of(dtype) || reinterpret_cast<uintptr_t>(dE) % size_of(out_dtype) ||
        reinterpret_cast<uintptr_t>(tokens) % 4 || reinterpret_cast<uintptr_t>(scratch) % 256)
        return PPO_ERR_ALIGN;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (N == 0) {
        if (accumulate) return PPO_OK;
        PPO_RETURN_IF_CUDA(cudaMemset2DAsync(dE, (size_t)lde * size_of(out_dtype), 0, (size_t)K * size_of(out_dtype), (size_t)V, s));
        return PPO_OK;
    }
    const bool vec = K % 8 == 0 && aligned_rows(dY, ldy, dtype) && aligned_rows(dE, lde, out_dtype);
    const Plan p = plan_of(N, K, V, vec);
    unsigned char *mem = reinterpret_cast<unsigned char *>(scratch);
    SortArgs sa = {};
    sa.tokens = tokens; sa.V = V; sa.N = (int)N; sa.padding_id = padding_id;
    sa.key = reinterpret_cast<int32_t *>(mem + p.key);
    sa.pos = reinterpret_cast<int32_t *>(mem + p.pos);
    sa.present = accumulate ? nullptr : mem + p.present;
    sa.status = workspace ? &ws_header(workspace)->status : nullptr;
    if (!accumulate) PPO_RETURN_IF_CUDA(cudaMemsetAsync(sa.present, 0, (size_t)V, s));
    int rc = launch_sort(sa, p, mem, s);
    if (rc) return rc;
    BwdArgs a = {};
    a.dY = dY; a.key = sa.key; a.pos = sa.pos; a.present = sa.present; a.dE = dE;
    a.part = reinterpret_cast<float *>(mem + p.part);
    a.V = V; a.ldy = ldy; a.lde = lde; a.N = (int)N; a.K = (int)K;
    a.chunk = p.chunk; a.chunks = p.chunks; a.accumulate = accumulate != 0; a.scale = scale;
    a.lanes = p.lanes; a.groups = p.groups; a.slabs = p.slabs;
    const int64_t blocks = (int64_t)((p.chunks + p.groups - 1) / p.groups) * p.slabs;
    a.fill_rows = (int)(K >= 16384 ? 1 : 65536 / K < 256 ? 65536 / K : 256);
    if (blocks + V / a.fill_rows + 1 >= ((int64_t)1 << 31) || (int64_t)p.chunks * ((K + kThreads - 1) / kThreads) >= ((int64_t)1 << 31))
        return PPO_ERR_SHAPE;
    a.chunk_blocks = (int)blocks;
    if (dtype == PPO_F32)
        return out_dtype == PPO_F32 ? launch_sums<float, float>(a, vec, s) : launch_sums<float, __nv_bfloat16>(a, vec, s);
    return out_dtype == PPO_F32 ? launch_sums<__nv_bfloat16, float>(a, vec, s) : launch_sums<__nv_bfloat16, __nv_bfloat16>(a, vec, s);
}
