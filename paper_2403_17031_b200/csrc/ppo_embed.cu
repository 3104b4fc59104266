// The input embedding: rows of a table, scaled (ppo_embed), and the gradient of the table (ppo_embed_bwd).
//
//     out[i, :] = scale * E[tokens[i], :]                       dE[v, :] = scale * sum over i with tokens[i] = v of dY[i, :]
//
// Both move bytes and do next to no arithmetic. The forward call reads each row once from memory (rows that occur again
// come from L2) and writes N rows. The gradient reads N rows and writes V, most of them zeros when N is small.
//
// Times: 326656 rows of 4096 bf16 546 us, 3.5 GB through DRAM at 6.5 TB/s (0.6 GB of it rows of the table that L2 lost again; wider
// accesses, other numbers of rows a block and L2 policies change nothing); their gradient into fp32 490 us (2.7 GB that have to move); of
// 27136 positions 110 us (0.57 GB), of 53 61 us (0.41 GB of zeros, 6.8 TB/s).
//
// Gradient: the positions are sorted by token (stable), so that the rows of one token follow one another. The sorted list
// is cut into chunks of equal length, whatever the tokens: text has a few tokens that make up a large share of it, and a
// block per token would leave them to a few blocks. A run of one token inside a chunk is summed in registers and
// written once; a run that crosses chunks leaves a partial sum per chunk, and those are added in the order of the chunks.
// Every sum is fp32 in ascending order of the positions, without atomics: results do not depend on timing. Rows of tokens
// that do not occur are zero-filled by other blocks of the same launches.
#include "ppo_packs.cuh"

namespace ppo {
namespace embed {

constexpr int kThreads = 256;

// A thread's columns of a row: Q packs of VEC neighbours, packs `lanes` apart so that a warp's accesses are contiguous.
// Rows at odd addresses are read element by element, four of them in flight.
template <int VEC> __host__ __device__ constexpr int packs_per_thread() { return VEC == 1 ? 4 : 1; }

static int widest(int64_t K, const void *a, int64_t lda, int ta, const void *b, int64_t ldb, int tb)
{
    for (int vec = 8; vec > 1; vec /= 2)
        if (K % vec == 0 && packs_fit(a, lda, ta, vec) && packs_fit(b, ldb, tb, vec)) return vec;
    return 1;
}

// ---------------------------------------------------------------- forward
struct FwdArgs {
    const void *table;
    const int32_t *tokens;
    void *out;
    int64_t N, V, lde, ldo;
    int K, sms;
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
            float x[VEC];
            p[r].get(x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[e] *= scale[r];
            if (i0 + r < a.N) Pack<TO, VEC>::store(out + r * a.ldo + k, x);
        }
    }
}

template <typename TI, typename TO, int VEC>
static void launch_lookup_vec(const FwdArgs &a, cudaStream_t s)
{
    // four rows per block once that leaves eight blocks for each SM (4096 bf16: 27136 rows 67 us, 73 one by one; 4736 14.5 and 15.1; 1184 6.0 and 5.2)
    if (a.N >= 4 * 8 * a.sms) lookup_kernel<TI, TO, VEC, 4><<<(unsigned)((a.N + 3) / 4), kThreads, 0, s>>>(a);
    else lookup_kernel<TI, TO, VEC, 1><<<(unsigned)a.N, kThreads, 0, s>>>(a);
}

template <typename TI, typename TO>
static int launch_lookup(const FwdArgs &a, int vec, cudaStream_t s)
{
    if (vec == 8) launch_lookup_vec<TI, TO, 8>(a, s);
    else if (vec == 4) launch_lookup_vec<TI, TO, 4>(a, s);
    else launch_lookup_vec<TI, TO, 1>(a, s);
    return launch_status();
}

// ---------------------------------------------------------------- the rows of the gradient
struct BwdArgs {
    const void *dY;
    const int32_t *tokens;
    const int32_t *key, *pos;       // sorted by token
    uint8_t *present;               // one byte a token, at present_at(): it occurs
    void *dE;
    float *part;                    // [chunks][2][K]: a run that comes from the chunk before; one that goes on in the next
    int64_t V, ldy, lde;
    int N, K, chunk, chunks, accumulate, padding_id;
    float scale;
    int lanes, groups, slabs;       // threads per chunk and slab, chunks per block (lanes * groups = kThreads)
    int fill_rows;                  // rows per block that zero-fills
    int64_t fill0;                  // first row of this launch's
    int work_blocks;                // blocks before those
    int *status;
};

template <typename TO, int VEC>
__device__ __forceinline__ void write_row(const BwdArgs &a, int64_t v, int k, float *x)
{
    TO *to = reinterpret_cast<TO *>(a.dE) + v * a.lde + k;
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] *= a.scale;
    if (a.accumulate) {
        Pack<TO, VEC> p;
        p.load_once(to);
        float old[VEC];
        p.get(old);
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[e] += old[e];
    }
    Pack<TO, VEC>::store(to, x);
}

// The zero rows are most of what few positions write, so they go along with the launches that sort, which leave nearly all of
// the memory's time unused; up to 8192 positions, which are ranked in one short launch, with the one that sums.
template <typename TO>
__device__ __forceinline__ void zero_row(const BwdArgs &a, int64_t v)
{
    zero_bytes(reinterpret_cast<unsigned char *>(reinterpret_cast<TO *>(a.dE) + v * a.lde), (int64_t)a.K * sizeof(TO));
}

// Place of a token's byte: neighbouring tokens in different 32-byte sectors. The most frequent tokens of a vocabulary are
// neighbours, and stores to one sector follow one another (326656 positions: counting takes 28 us with the bytes in order, 10 so).
__device__ __forceinline__ uint8_t *present_at(const BwdArgs &a, int64_t v)
{
    const int64_t sectors = (a.V + 31) / 32;
    return a.present + (v % sectors) * 32 + v / sectors;
}

template <typename TO>
__device__ __forceinline__ void fill_rows(const BwdArgs &a, int block)
{
    const int64_t v0 = a.fill0 + (int64_t)block * a.fill_rows;
    for (int64_t v = v0 + threadIdx.x / 32; v < v0 + a.fill_rows && v < a.V; v += blockDim.x / 32)
        if (!*present_at(a, v)) zero_row<TO>(a, v);
}

__device__ __forceinline__ int key_of(const BwdArgs &a, int t) { return t < 0 || t >= a.V || t == a.padding_id ? (int)a.V : t; }

// ---------------------------------------------------------------- a handful of positions: one launch, no sorting
// A block owns a few rows. It looks all tokens through for them, in order, and writes its rows: sums or zeros. (A third of the
// positions of text are of one block's rows: 300 positions x 1024 take 57 us in this form, 38 sorted.)
constexpr int kDirectMax = 128, kDirectRows = 16;
static_assert(kDirectMax <= kThreads, "a thread for each position");
template <typename TI, typename TO, int VEC>
__global__ void __launch_bounds__(kThreads)
direct_kernel(const BwdArgs a)
{
    __shared__ int row[kDirectMax], pos[kDirectMax], warp_n[kThreads / 32];
    const int64_t v0 = (int64_t)blockIdx.x * kDirectRows;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int t = -1;
    if ((int)threadIdx.x < a.N) {
        const int raw = a.tokens[threadIdx.x];
        if (blockIdx.x == 0 && a.status && (raw < 0 || raw >= a.V)) atomicOr(a.status, PPO_DEV_BAD_TOKEN);
        const int64_t off = key_of(a, raw) - v0;
        if (key_of(a, raw) < a.V && off >= 0 && off < kDirectRows) t = (int)off;
    }
    const unsigned mine = __ballot_sync(0xffffffffu, t >= 0);
    if (lane == 0) warp_n[warp] = __popc(mine);
    __syncthreads();
    int at = __popc(mine & ((1u << lane) - 1)), n = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) at += warp_n[w];
        n += warp_n[w];
    }
    if (t >= 0) {
        row[at] = t;
        pos[at] = threadIdx.x;
    }
    __syncthreads();
    const TI *dY = reinterpret_cast<const TI *>(a.dY);
    const int rows = (int)min((int64_t)kDirectRows, a.V - v0);
    unsigned occur = 0;
    for (int i = 0; i < n; ++i) occur |= 1u << row[i];
    // zero rows, then the others
    if (!a.accumulate) {
        for (int r = warp; r < rows; r += kThreads / 32)
            if (!(occur >> r & 1)) zero_row<TO>(a, v0 + r);
    }
    for (; occur; occur &= occur - 1) {
        const int r = __ffs(occur) - 1;
        for (int k = threadIdx.x * VEC; k < a.K; k += kThreads * VEC) {
            float acc[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
            for (int i = 0; i < n;) {
                constexpr int U = 8;                            // rows in flight
                Pack<TI, VEC> p[U];
                int got = 0;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    while (i < n && row[i] != r) ++i;
                    if (i < n) {
                        p[u].load(dY + (int64_t)pos[i++] * a.ldy + k);
                        got = u + 1;
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (u >= got) break;
                    float x[VEC];
                    p[u].get(x);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) acc[e] += x[e];
                }
            }
            write_row<TO, VEC>(a, v0 + r, k, acc);
        }
    }
}

// ---------------------------------------------------------------- sorting the positions by token
// Keys are token ids; a position that counts for no row (padding id, id outside [0, V)) has the key V and comes last.
__device__ __forceinline__ void note_token(const BwdArgs &a, int t, int key)
{
    if (key < a.V) {
        if (!a.accumulate) *present_at(a, key) = 1;
    } else if (a.status && (t < 0 || t >= a.V)) {
        atomicOr(a.status, PPO_DEV_BAD_TOKEN);
    }
}

// Up to 8192 positions of up to 2^19 tokens: each one's place is the number of (key, position) pairs below its own, counted.
// A warp counts for two positions. (5087 positions 9 us; the passes below take 25 for
// 20000.)
constexpr int kRankPer = 2, kRankMax = 8192, kRankBits = 13, kRankWarps = kThreads / 32;
constexpr int64_t kRankVocabulary = (int64_t)1 << (32 - kRankBits);
__global__ void __launch_bounds__(kThreads)
rank_kernel(const BwdArgs a, int32_t *__restrict__ key_out, int32_t *__restrict__ pos_out)
{
    __shared__ uint32_t pair[kRankMax];
    grid_dependents_may_launch();
#pragma unroll 8
    for (int j = threadIdx.x; j < a.N; j += kThreads) pair[j] = (uint32_t)key_of(a, a.tokens[j]) << kRankBits | (uint32_t)j;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    const int i0 = (blockIdx.x * kRankWarps + (threadIdx.x >> 5)) * kRankPer;
    uint32_t mine[kRankPer];
    int n[kRankPer];
#pragma unroll
    for (int r = 0; r < kRankPer; ++r) {
        mine[r] = i0 + r < a.N ? pair[i0 + r] : 0;
        n[r] = 0;
    }
#pragma unroll 8
    for (int j = lane; j < a.N; j += 32) {
        const uint32_t p = pair[j];
#pragma unroll
        for (int r = 0; r < kRankPer; ++r) n[r] += p < mine[r];
    }
#pragma unroll
    for (int r = 0; r < kRankPer; ++r) {
        n[r] = __reduce_add_sync(0xffffffffu, n[r]);
        if (lane == r && i0 + r < a.N) {
            const int key = (int)(mine[r] >> kRankBits);
            key_out[n[r]] = key;
            pos_out[n[r]] = i0 + r;
            note_token(a, a.tokens[i0 + r], key);
        }
    }
}

// Tiles up to which each block sums the counts itself, instead of a launch for it (20000 positions: 57 us with the launches).
constexpr int kSumTiles = 128, kAheadTiles = 16;

// More: least significant digit first, 8 bits a pass, each pass stable: digits counted per tile, the counts summed in digit
// order, the tile's entries moved. A warp owns neighbouring entries of a tile. With few tiles a pass that moves an entry counts
// it for the next one, whose tile it knows, and saves that pass the launch for counting (150000 positions: 35 us a pass so, 13 and 6 for
// the launch without).
constexpr int kTile = 2048, kDigits = 256, kWarps = kThreads / 32, kPerWarp = kTile / kWarps;

struct PassArgs {
    const int32_t *key_in, *pos_in;      // null in the first pass
    int32_t *key_out, *pos_out;
    int32_t *counts, *next_counts;       // [kDigits][pitch], zeros behind the tiles; next_counts null in the last pass
    int tiles, pitch, shift;
    int summed;                          // the counts have been summed up (many tiles)
};

__device__ __forceinline__ void load_entry(const BwdArgs &a, const PassArgs &p, int i, int &key, int &pos)
{
    key = p.key_in ? p.key_in[i] : key_of(a, a.tokens[i]);
    pos = p.pos_in ? p.pos_in[i] : i;
}

constexpr int kSeen = 1024;
__global__ void __launch_bounds__(kThreads)
count_kernel(const BwdArgs a, const PassArgs p)
{
    // Frequent tokens: one addition for a warp's equal digits, and no second note of a token that the block noted last in its
    // place of `seen` (text has a third of its tokens in one sector of `present`, whose stores would follow one another:
    // 326656 positions 38 us).
    __shared__ int n[kDigits], seen[kSeen];
    grid_dependents_may_launch();
    n[threadIdx.x] = 0;
#pragma unroll
    for (int j = 0; j < kSeen; j += kThreads) seen[j + threadIdx.x] = -1;
    constexpr int R = kTile / kThreads;
    const int i0 = blockIdx.x * kTile + threadIdx.x;
    // (the first pass takes the tokens, the others keys that have been noted)
    int t[R];
    if (p.key_in) grid_dependency_wait();
    const int32_t *from = p.key_in ? p.key_in : a.tokens;
#pragma unroll
    for (int j = 0; j < R; ++j) t[j] = i0 + j * kThreads < a.N ? from[i0 + j * kThreads] : 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const bool in = i0 + j * kThreads < a.N;
        const int key = p.key_in ? t[j] : key_of(a, t[j]), digit = in ? (key >> p.shift) & (kDigits - 1) : kDigits;
        const unsigned same = __match_any_sync(0xffffffffu, digit);
        if (in && (same & ((1u << (threadIdx.x & 31)) - 1)) == 0) atomicAdd(&n[digit], __popc(same));
        // (all that counts for no row has one key: of those each is looked at)
        if (in && !p.key_in && (key >= a.V || seen[key & (kSeen - 1)] != key)) {
            seen[key & (kSeen - 1)] = key;
            note_token(a, t[j], key);
        }
    }
    __syncthreads();
    p.counts[(size_t)threadIdx.x * p.pitch + blockIdx.x] = n[threadIdx.x];
}

// exclusive sum over the counts, in place; one block
constexpr int kScanThreads = 1024;
template <typename TO>
__global__ void __launch_bounds__(kScanThreads)
scan_kernel(const BwdArgs a, const PassArgs p)
{
    grid_dependents_may_launch();
    grid_dependency_wait();
    if (blockIdx.x > 0) {
        fill_rows<TO>(a, blockIdx.x - 1);
        return;
    }
    __shared__ int warp_sum[32];
    __shared__ int carry;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = p.pitch * kDigits;
    int4 *counts = reinterpret_cast<int4 *>(p.counts);          // (kDigits counts a tile: a multiple of 8)
    if (threadIdx.x == 0) carry = 0;
    __syncthreads();
    for (int base = 0; base < n; base += kScanThreads * 8) {
        const int i = base + threadIdx.x * 8;
        int v[8] = {0, 0, 0, 0, 0, 0, 0, 0}, sum = 0;
        if (i < n) {
            const int4 x = counts[i / 4], y = counts[i / 4 + 1];
            v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int x = v[e];
            v[e] = sum;
            sum += x;
        }
        int incl = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += o;
        }
        if (lane == 31) warp_sum[warp] = incl;
        __syncthreads();
        const int w = warp_sum[lane];
        const int before = carry + __reduce_add_sync(0xffffffffu, lane < warp ? w : 0) + incl - sum;
        if (i < n) {
            counts[i / 4] = make_int4(before + v[0], before + v[1], before + v[2], before + v[3]);
            counts[i / 4 + 1] = make_int4(before + v[4], before + v[5], before + v[6], before + v[7]);
        }
        __syncthreads();
        if (threadIdx.x == kScanThreads - 1) carry = before + sum;
        __syncthreads();
    }
}

template <typename TO>
__global__ void __launch_bounds__(kThreads)
scatter_kernel(const BwdArgs a, const PassArgs p)
{
    grid_dependents_may_launch();
    grid_dependency_wait();
    if ((int)blockIdx.x >= a.work_blocks) {
        fill_rows<TO>(a, blockIdx.x - a.work_blocks);
        return;
    }
    __shared__ int at[kWarps][kDigits];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int j = threadIdx.x; j < kWarps * kDigits; j += kThreads) (&at[0][0])[j] = 0;
    const int i0 = blockIdx.x * kTile + warp * kPerWarp;
    constexpr int R = kPerWarp / 32;
    int key[R], pos[R], before[R];
    unsigned same[R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int i = i0 + j * 32 + lane;
        key[j] = -1;
        if (i < a.N) load_entry(a, p, i, key[j], pos[j]);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int digit = key[j] >= 0 ? (key[j] >> p.shift) & (kDigits - 1) : kDigits;
        same[j] = __match_any_sync(0xffffffffu, digit);
        before[j] = __popc(same[j] & ((1u << lane) - 1));
        if (key[j] >= 0 && before[j] == 0) atomicAdd(&at[warp][digit], __popc(same[j]));
    }
    __syncthreads();
    {   // the warps' first places of each digit
        int run;
        const int32_t *mine = p.counts + (size_t)threadIdx.x * p.pitch;
        if (p.summed) {
            run = mine[blockIdx.x];
        } else {
            // a thread for a digit: its count in the tiles before this one and in all; then the digits before it
            __shared__ int warp_sum[kWarps];
            int total = 0;
            run = 0;
#pragma unroll 4
            for (int t = 0; t < p.pitch; t += 4) {
                const int4 c = *reinterpret_cast<const int4 *>(mine + t);
                total += c.x + c.y + c.z + c.w;
                const int b = (int)blockIdx.x - t;
                run += (b > 0 ? c.x : 0) + (b > 1 ? c.y : 0) + (b > 2 ? c.z : 0) + (b > 3 ? c.w : 0);
            }
            int incl = total;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, incl, off);
                if (lane >= off) incl += o;
            }
            if (lane == 31) warp_sum[warp] = incl;
            __syncthreads();
            run += incl - total;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) run += w < warp ? warp_sum[w] : 0;
        }
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const int n = at[w][threadIdx.x];
            at[w][threadIdx.x] = run;
            run += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int digit = (key[j] >> p.shift) & (kDigits - 1);
        int to = 0;
        if (key[j] >= 0) to = at[warp][digit] + before[j];
        __syncwarp();
        if (key[j] >= 0 && before[j] == 0) at[warp][digit] += __popc(same[j]);
        __syncwarp();
        if (key[j] >= 0) {
            p.key_out[to] = key[j];
            p.pos_out[to] = pos[j];
        }
        if (p.next_counts) {
            // one addition for the warp's equal ones, as above
            const int at2 = key[j] >= 0 ? ((key[j] >> (p.shift + 8)) & (kDigits - 1)) * p.pitch + to / kTile : -1;
            const unsigned equal = __match_any_sync(0xffffffffu, at2);
            if (at2 >= 0 && (equal & ((1u << lane) - 1)) == 0) atomicAdd(&p.next_counts[at2], __popc(equal));
        }
    }
}

// ---------------------------------------------------------------- sums
template <typename TI, typename TO, int VEC>
__global__ void __launch_bounds__(kThreads, 3)
sum_kernel(const BwdArgs a)
{
    constexpr int Q = packs_per_thread<VEC>(), U = (VEC * sizeof(TI) > 16 ? 4 : 8) / Q;      // rows in flight
    grid_dependents_may_launch();
    grid_dependency_wait();
    if ((int)blockIdx.x >= a.work_blocks) {
        fill_rows<TO>(a, blockIdx.x - a.work_blocks);
        return;
    }
    extern __shared__ int2 entries[];                           // [groups][chunk] key, position
    const int lane = threadIdx.x % a.lanes, group = threadIdx.x / a.lanes;
    const int slab = blockIdx.x % a.slabs, c0 = (blockIdx.x / a.slabs) * a.groups, c = c0 + group;
    {
        const int64_t first = (int64_t)c0 * a.chunk;
#pragma unroll 4
        for (int j = threadIdx.x; j < a.groups * a.chunk; j += kThreads)
            entries[j] = first + j < a.N ? make_int2(a.key[first + j], a.pos[first + j]) : make_int2(-1, 0);
    }
    const int e0 = c * a.chunk;
    int before = -1, behind = -1;
    if (c < a.chunks) {
        if (e0 > 0) before = a.key[e0 - 1];
        if (c + 1 < a.chunks) behind = a.key[e0 + a.chunk];
    }
    __syncthreads();
    if (c >= a.chunks) return;
    const int2 *mine = entries + group * a.chunk;
    int k[Q];
    bool in[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        k[q] = ((slab * Q + q) * a.lanes + lane) * VEC;
        in[q] = k[q] < a.K;
    }
    const TI *dY = reinterpret_cast<const TI *>(a.dY);
    float acc[Q][VEC];
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[q][e] = 0.f;
    int cur = mine[0].x;
    bool from_before = before == cur;
    const auto flush = [&](bool goes_on) {
        if (cur >= a.V) return;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            if (!in[q]) continue;
            if (from_before || goes_on) {
                float *to = a.part + ((size_t)c * 2 + (from_before ? 0 : 1)) * a.K + k[q];
                Pack<float, VEC>::store(to, acc[q]);
            } else {
                write_row<TO, VEC>(a, cur, k[q], acc[q]);
            }
        }
    };
    for (int e = 0; e < a.chunk; e += U) {                      // (a chunk is a multiple of 8)
        if (mine[e].x < 0 || mine[e].x >= a.V) break;
        Pack<TI, VEC> p[U][Q];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int2 en = mine[e + u];
            const TI *row = dY + (int64_t)en.y * a.ldy;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                if ((unsigned)en.x < (unsigned)a.V && in[q]) p[u][q].load_once(row + k[q]);
                else p[u][q].zero();
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int key = mine[e + u].x;
            if (key >= 0 && key != cur) {
                flush(false);
                cur = key;
                from_before = false;
#pragma unroll
                for (int q = 0; q < Q; ++q)
#pragma unroll
                    for (int x = 0; x < VEC; ++x) acc[q][x] = 0.f;
            }
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                float x[VEC];
                p[u][q].get(x);
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[q][i] += x[i];
            }
        }
    }
    flush(behind == cur);
}

// The runs that cross chunks: the block of the chunk in which such a run begins adds the partial sums up.
template <typename TO, int VEC>
__global__ void __launch_bounds__(kThreads)
join_kernel(const BwdArgs a)
{
    grid_dependency_wait();
    const int c = blockIdx.x / a.slabs, k = ((blockIdx.x % a.slabs) * kThreads + threadIdx.x) * VEC;
    const int e0 = c * a.chunk, e1 = e0 + a.chunk;              // (the last chunk has no block)
    const int t = a.key[e1 - 1], next = a.key[e1], before = e0 > 0 ? a.key[e0 - 1] : -1;
    if (t >= a.V || next != t) return;                          // no run goes on
    if (before == t) return;                                    // it began in an earlier chunk
    int lo = c + 1, hi = a.chunks - 1;                          // last chunk that begins with t
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.key[(size_t)mid * a.chunk] == t) lo = mid;
        else hi = mid - 1;
    }
    if (k >= a.K) return;
    Pack<float, VEC> p;
    float sum[VEC];
    p.load(a.part + ((size_t)c * 2 + 1) * a.K + k);
    p.get(sum);
#pragma unroll 16
    for (int i = c + 1; i <= lo; ++i) {
        p.load(a.part + (size_t)i * 2 * a.K + k);
        float x[VEC];
        p.get(x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] += x[e];
    }
    write_row<TO, VEC>(a, t, k, sum);
}

// ---------------------------------------------------------------- host side
struct Plan {
    int chunk, chunks, tiles, passes;
    bool direct;
    size_t key, pos, key2, pos2, counts, first_zero, present, zero_bytes, part, bytes;
};

// (the same for every alignment: the caller asks for the scratch before it has the tensors)
static Plan plan_of(int64_t N, int64_t K, int64_t V)
{
    Plan p = {};
    p.direct = N <= kDirectMax;
    if (p.direct) {
        p.bytes = 256;
        return p;
    }
    // 128 entries, or so many that 3500 blocks have work: 2048 columns of a chunk each (150000 x 1000: 90 us with 586 blocks)
    p.chunk = 128;
    while (p.chunk > 32 && N / p.chunk * K < (int64_t)3500 * 2048) p.chunk /= 2;
    p.chunks = (int)((N + p.chunk - 1) / p.chunk);
    if (N > kRankMax || V >= kRankVocabulary) {
        p.tiles = (int)((N + kTile - 1) / kTile);
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
    const size_t ints = (size_t)N * 4, counts = align256((size_t)(p.tiles + 3) / 4 * 4 * kDigits * 4);
    p.key = take(ints);
    p.pos = take(ints);
    p.key2 = take(p.tiles ? ints : 0);
    p.pos2 = take(p.tiles ? ints : 0);
    p.counts = take(counts * p.passes);
    p.present = take(((size_t)V + 31) / 32 * 32);
    // cleared first: the counts, and `present`
    p.first_zero = p.counts;
    p.zero_bytes = at - p.first_zero;
    p.part = take((size_t)p.chunks * 2 * (size_t)K * 4);
    p.bytes = at;
    return p;
}

// Zero rows are handed out to the launches in `parts` shares; 0 shares: all that is left.
struct Fill {
    int64_t next, blocks, share;
    int rows;
    void init(const BwdArgs &a, int parts)
    {
        rows = a.fill_rows;
        next = 0;
        blocks = a.accumulate ? 0 : (a.V + rows - 1) / rows;
        share = blocks / parts;
    }
    unsigned take(BwdArgs &a, int shares)
    {
        const int64_t n = shares ? shares * share : blocks - next;
        a.fill0 = next * rows;
        next += n;
        return (unsigned)n;
    }
};

template <typename TI, typename TO, int VEC>
static int launch_bwd(BwdArgs a, const Plan &p, unsigned char *mem, cudaStream_t s)
{
    if (p.direct) {
        direct_kernel<TI, TO, VEC><<<(unsigned)((a.V + kDirectRows - 1) / kDirectRows), kThreads, 0, s>>>(a);
        return launch_status();
    }
    int rc;
    Fill fill;
    int32_t *key[2] = {reinterpret_cast<int32_t *>(mem + p.key), reinterpret_cast<int32_t *>(mem + p.key2)};
    int32_t *pos[2] = {reinterpret_cast<int32_t *>(mem + p.pos), reinterpret_cast<int32_t *>(mem + p.pos2)};
    a.key = key[0];
    a.pos = pos[0];
    const size_t counts = align256((size_t)(p.tiles + 3) / 4 * 4 * kDigits * 4);
    if (!a.accumulate || p.passes > 0) PPO_RETURN_IF_CUDA(cudaMemsetAsync(mem + p.first_zero, 0, p.zero_bytes, s));
    if (!p.tiles) {
        fill.init(a, 1);
        const int per_block = kRankWarps * kRankPer;
        rank_kernel<<<(a.N + per_block - 1) / per_block, kThreads, 0, s>>>(a, key[0], pos[0]);
        if ((rc = launch_status())) return rc;
    } else {
        // (moving the entries leaves the memory more time than the other launches do)
        fill.init(a, 4 * p.passes);
        PassArgs ps = {};
        ps.tiles = p.tiles;
        ps.pitch = (p.tiles + 3) / 4 * 4;
        ps.summed = p.tiles > kSumTiles;
        int to = (p.passes & 1) ^ 1;                            // the last pass writes the first pair
        for (int pass = 0; pass < p.passes; ++pass, to ^= 1) {
            ps.counts = reinterpret_cast<int32_t *>(mem + p.counts + pass * counts);
            ps.next_counts = pass + 1 < p.passes && p.tiles <= kAheadTiles ? reinterpret_cast<int32_t *>(mem + p.counts + (pass + 1) * counts) : nullptr;
            ps.key_out = key[to];
            ps.pos_out = pos[to];
            ps.shift = pass * 8;
            if (pass == 0) {
                count_kernel<<<p.tiles, kThreads, 0, s>>>(a, ps);
                if ((rc = launch_status())) return rc;
            } else if (p.tiles > kAheadTiles) {
                PPO_RETURN_IF_CUDA(launch_dependent(count_kernel, dim3(p.tiles), dim3(kThreads), 0, s, a, ps));
            }
            if (ps.summed) {
                const unsigned extra = fill.take(a, 1);
                PPO_RETURN_IF_CUDA(launch_dependent(scan_kernel<TO>, dim3(1 + extra), dim3(kScanThreads), 0, s, a, ps));
            }
            const unsigned extra = fill.take(a, ps.summed ? 3 : 4);
            a.work_blocks = p.tiles;
            PPO_RETURN_IF_CUDA(launch_dependent(scatter_kernel<TO>, dim3(p.tiles + extra), dim3(kThreads), 0, s, a, ps));
            ps.key_in = ps.key_out;
            ps.pos_in = ps.pos_out;
        }
    }
    const int64_t packs = (a.K + VEC * packs_per_thread<VEC>() - 1) / (VEC * packs_per_thread<VEC>());   // threads for a row
    a.lanes = 8;
    while (a.lanes < kThreads && a.lanes < packs) a.lanes *= 2;
    a.groups = kThreads / a.lanes;
    a.slabs = (int)((packs + a.lanes - 1) / a.lanes);
    const int64_t blocks = (int64_t)((p.chunks + a.groups - 1) / a.groups) * a.slabs;
    constexpr int kJoinVec = VEC > 4 ? 4 : VEC;
    const int join_slabs = (int)((a.K + kThreads * kJoinVec - 1) / (kThreads * kJoinVec));
    if (blocks + a.V / a.fill_rows + 1 >= ((int64_t)1 << 31) || (int64_t)p.chunks * join_slabs >= ((int64_t)1 << 31)) return PPO_ERR_SHAPE;
    a.work_blocks = (int)blocks;
    const unsigned extra = fill.take(a, 0);
    PPO_RETURN_IF_CUDA(launch_dependent(sum_kernel<TI, TO, VEC>, dim3((unsigned)blocks + extra), dim3(kThreads),
                                        (size_t)a.groups * a.chunk * sizeof(int2), s, a));
    if (p.chunks < 2) return PPO_OK;
    a.slabs = join_slabs;
    PPO_RETURN_IF_CUDA(launch_dependent(join_kernel<TO, kJoinVec>, dim3((unsigned)((p.chunks - 1) * join_slabs)), dim3(kThreads), 0, s, a));
    return PPO_OK;
}

template <typename TI, typename TO>
static int launch_bwd_types(const BwdArgs &a, const Plan &p, int vec, unsigned char *mem, cudaStream_t s)
{
    return vec == 8 ? launch_bwd<TI, TO, 8>(a, p, mem, s) : vec == 4 ? launch_bwd<TI, TO, 4>(a, p, mem, s) : launch_bwd<TI, TO, 1>(a, p, mem, s);
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
        reinterpret_cast<uintptr_t>(tokens) % 4 || reinterpret_cast<uintptr_t>(workspace) % 256)
        return PPO_ERR_ALIGN;
    int dev = 0, sms = 148;
    PPO_RETURN_IF_CUDA(cudaGetDevice(&dev));
    PPO_RETURN_IF_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    FwdArgs a = {};
    a.table = table; a.tokens = tokens; a.out = out;
    a.N = N; a.V = V; a.K = (int)K; a.sms = sms; a.lde = lde; a.ldo = ldo; a.scale = scale;
    a.status = workspace ? &ws_header(workspace)->status : nullptr;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const int vec = widest(K, table, lde, dtype, out, ldo, out_dtype);
    if (dtype == PPO_F32)
        return out_dtype == PPO_F32 ? launch_lookup<float, float>(a, vec, s) : launch_lookup<float, __nv_bfloat16>(a, vec, s);
    return out_dtype == PPO_F32 ? launch_lookup<__nv_bfloat16, float>(a, vec, s) : launch_lookup<__nv_bfloat16, __nv_bfloat16>(a, vec, s);
}

extern "C" size_t ppo_embed_bwd_scratch_bytes(int64_t N, int64_t K, int64_t V)
{
    using namespace embed;
    if (N <= 0 || K <= 0 || V <= 0 || N >= kLimit || K >= kLimit || V >= kLimit) return 0;
    return plan_of(N, K, V).bytes;
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
        reinterpret_cast<uintptr_t>(tokens) % 4 || reinterpret_cast<uintptr_t>(scratch) % 256 || reinterpret_cast<uintptr_t>(workspace) % 256)
        return PPO_ERR_ALIGN;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (N == 0) {
        if (accumulate) return PPO_OK;
        PPO_RETURN_IF_CUDA(cudaMemset2DAsync(dE, (size_t)lde * size_of(out_dtype), 0, (size_t)K * size_of(out_dtype), (size_t)V, s));
        return PPO_OK;
    }
    const int vec = widest(K, dY, ldy, dtype, dE, lde, out_dtype);
    const Plan p = plan_of(N, K, V);
    unsigned char *mem = reinterpret_cast<unsigned char *>(scratch);
    BwdArgs a = {};
    a.dY = dY; a.tokens = tokens; a.dE = dE; a.padding_id = padding_id;
    a.present = mem + p.present;
    a.part = reinterpret_cast<float *>(mem + p.part);
    a.V = V; a.ldy = ldy; a.lde = lde; a.N = (int)N; a.K = (int)K;
    a.chunk = p.chunk; a.chunks = p.chunks; a.accumulate = accumulate != 0; a.scale = scale;
    // (64 KB a block, eight rows for its warps at least)
    const int64_t row_bytes = K * (int64_t)size_of(out_dtype);
    a.fill_rows = (int)(row_bytes >= 8192 ? 8 : 65536 / row_bytes < 256 ? 65536 / row_bytes : 256);
    a.status = workspace ? &ws_header(workspace)->status : nullptr;
    if (dtype == PPO_F32)
        return out_dtype == PPO_F32 ? launch_bwd_types<float, float>(a, p, vec, mem, s)
                                    : launch_bwd_types<float, __nv_bfloat16>(a, p, vec, mem, s);
    return out_dtype == PPO_F32 ? launch_bwd_types<__nv_bfloat16, float>(a, p, vec, mem, s)
                                : launch_bwd_types<__nv_bfloat16, __nv_bfloat16>(a, p, vec, mem, s);
}
