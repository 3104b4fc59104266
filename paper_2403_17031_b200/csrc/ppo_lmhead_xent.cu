// Cross entropy at the LM head with both gradients (ppo_lmhead_xent), without a matrix of rows x vocabulary in memory:
//     z = H W / tau,   nll_r = lse_r - z[r, label_r],   loss = sum of nll over the real rows / n
//     D = scale / (n tau) * (softmax(z) - onehot(label)),   dH = D W^T,   dW = H^T D
//
// The rows go through in pieces, three products each (6 K V flops a row: nothing is formed twice):
//   1  U = 2^(y - ref), y = z log2(e), from the accumulators, stored once in bf16 for the piece. The softmax' sum is not
//      known while the tiles are formed, so U is left unnormalised: with S_r = sum_j U_rj the gradient is
//          D_r = a_r (U_r - S_r onehot),   a_r = scale / (n tau S_r),
//      a factor per row, which the other two products can take on their own: U gets S subtracted at the label (one element
//      a row), product 2 multiplies its rows by a_r in its epilogue, product 3 takes a_r H instead of H. No pass over a
//      piece of the logits is needed between the products.
//   2  dH = a (U' W^T)
//   3  dW = (a H)^T U', over all pieces: fp32 sums in scratch, tile by tile in the order in which the epilogue holds them
// A row's reference is set before product 1, from the mean of 64 neighbouring logits, and serves columns whose largest y lies between 32
// below and 96 above that mean: U and its sums stay inside fp32's (and bf16's) exponents, for logits of any size. 128 columns whose
// largest lies elsewhere move their own reference by multiples of 128; where a row's references differ, the columns with a
// smaller one are multiplied by 2^(difference), which is exact, before product 2.
//
// Roundings to 16 bits: U, a H, and the results. Statistics, sums and nll are fp32, the loss fp64. What the rounding of U
// would do to the gradients is kept small in three ways. S in the gradient is the sum of the rounded U, so that D is the
// gradient of a softmax whose probabilities are off by half a step each and still add up to 1: a direction that all columns
// of W share drops out of dH (logits far from 0 have one), as it should. U' at the label, about -S, is the largest element
// of its row by far; what its own rounding leaves, e = (U - S) - U', comes back in fp32: in product 2 as e W[:, label], in
// the epilogue, and in product 3 by a factor that makes a U' exact there (the row's other elements take that half step).
//
// Product kernel: persistent pairs of blocks (cta_group::2) on 256 x 256 tiles; per block one TMA producer warp (stages of
// 64 along the contraction, 128-byte swizzle), in the leader one issuer warp, eight epilogue warps that drain one 256-column
// accumulator while the next is formed. Operands are read as they lie in memory, K-major or MN-major, so that W may be
// stored [K, V] or [V, K].
#include "ppo_tcgen05.cuh"

namespace ppo {
namespace xent {

using namespace tc;

constexpr int kBM = 128, kTile = 256, kBlockK = 64, kStages = 5;
constexpr int kHalf = kBM * kBlockK * 2, kStage = 2 * kHalf, kBox = 64 * kBlockK * 2;    // bytes: a block's half of A or of B
constexpr int kEpiWarps = 8, kThreads = (4 + kEpiWarps) * 32;
constexpr int kStageOut = 32 * 128;                        // two per epilogue warp: 32 rows x 64 bf16
constexpr int kSmem = kStages * kStage + 2 * kEpiWarps * kStageOut + 1024;
constexpr int kChunk = 128;                                // columns with one reference
constexpr int kMaxPairs = 80;
constexpr int kTileFloats = kTile * kTile;
constexpr float kNoRef = -1.0e30f;
static_assert(kSmem <= 232448 - 1024, "shared memory of a block");

enum Product { kLogits = 1, kHidden = 2, kWeight = 3 };

struct Args {
    // rows of this piece: min(rows_max, max(0, *n_real - row0)), known on the device
    const int *n_real;
    int M, row0, rows_max;
    int dim_m, dim_n, dim_k;                               // result [dim_m, dim_n], contraction dim_k; the rows' one is an upper bound
    int gm, gn;
    int *status;
    // kLogits
    float c;                                               // log2(e) / tau
    const int32_t *labels, *order;                         // order[i]: the original row of real row i
    const float *base;                                     // [M] reference of real row i
    float *picked;                                         // [rows] accumulator at the label
    float4 *part;                                          // [rows][chunks] reference, sum, sum of the rounded values
    int chunks, store;
    // results
    __nv_bfloat16 *out;
    int64_t ldo;
    int bulk_cols;                                         // bulk stores take boxes that end at or before this column
    // kHidden
    const float2 *row_scale;                               // [rows] a, a e
    const __nv_bfloat16 *W;
    int64_t ldw;
    float *scratch;                                        // kHidden: parts of tiles cut along the contraction; kWeight: sums over the pieces
};

__device__ __forceinline__ int rows_of(const Args &a) { return max(0, min(a.rows_max, *a.n_real - a.row0)); }

// A wait that is skipped once one has run out: the block then reaches its end quickly, with the same control flow. Whoever
// has given up announces nothing any more, and an epilogue warp that has given up stores NaN.
__device__ __forceinline__ void wait_alive(bool &alive, unsigned long long *bar, uint32_t parity, int *status)
{
    if (alive) alive = wait(bar, parity, status);
}

// PPO_TEST_WITHHOLD_XENT (never defined in the product build): a test build in which 1: finished accumulators are never
// announced, 2: drained ones are not.
#ifndef PPO_TEST_WITHHOLD_XENT
#define PPO_TEST_WITHHOLD_XENT 0
#endif

struct Smem {
    unsigned long long full[kStages], empty[kStages], tmem_full[2], tmem_empty[2];
    uint32_t tmem_base;
};

// The pairs take tiles 0 .. n_whole in turn, whole. With `share` > 0 the other tiles, too few for all pairs, are cut along
// the contraction: end to end they are n_rest * kbs blocks, of which pair c takes share, from c * share on (at most two
// tiles), and join_kernel adds the parts up in the order of the pairs.
struct Plan {
    int m_tiles, n_tiles, n_whole, n_rest, share, kbs;
};

template <int PRODUCT>
__device__ __forceinline__ Plan plan_of(const Args &a, int rows, int pairs)
{
    Plan p;
    p.m_tiles = ((PRODUCT == kWeight ? a.dim_m : rows) + kTile - 1) / kTile;
    p.n_tiles = (a.dim_n + kTile - 1) / kTile;
    p.kbs = ((PRODUCT == kWeight ? rows : a.dim_k) + kBlockK - 1) / kBlockK;
    p.n_whole = p.m_tiles * p.n_tiles;
    p.n_rest = p.share = 0;
    if (PRODUCT == kWeight && rows == 0 && a.row0 > 0) p.n_whole = 0;      // nothing to add
    if (PRODUCT == kHidden) {
        // cut when that saves each pair 24 blocks of the contraction or more
        const int rest = p.n_whole % pairs, share = (int)(((int64_t)rest * p.kbs + pairs - 1) / pairs);
        if (rest > 0 && p.kbs - share >= 24) {
            p.n_rest = rest;
            p.n_whole -= rest;
            p.share = share;
        }
    }
    return p;
}

struct Work {
    int u, kb0, kb1;      // tile, blocks of the contraction
    int part;             // -1: whole; else which of the pair's parts
    int u_next, r, r_end;
    __device__ __forceinline__ void init(const Plan &p, int pair)
    {
        u_next = pair;
        r = min(pair * p.share, p.n_rest * p.kbs);
        r_end = min(r + p.share, p.n_rest * p.kbs);
        part = -1;
    }
    __device__ __forceinline__ bool next(const Plan &p, int pairs)
    {
        if (u_next < p.n_whole) {
            u = u_next;
            u_next += pairs;
            kb0 = 0;
            kb1 = p.kbs;
            return true;
        }
        if (r >= r_end) return false;
        const int t = r / p.kbs;
        u = p.n_whole + t;
        kb0 = r - t * p.kbs;
        kb1 = min(p.kbs, kb0 + r_end - r);
        r += kb1 - kb0;
        ++part;
        return true;
    }
};

// 32 rows x 64 bf16 from a warp's staging buffer (16-byte piece p of row r at p ^ (r & 7)) to rows out_row (lane r holds
// row r's, -1: none) at column n
__device__ __forceinline__ void store_rows(const unsigned char *stage, __nv_bfloat16 *out, int64_t ldo, int out_row, int n, int cols)
{
    const int lane = threadIdx.x & 31;
    if (reinterpret_cast<uintptr_t>(out) % 16 == 0 && ldo % 8 == 0 && n + 64 <= cols) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = i * 4 + (lane >> 3), p = lane & 7;
            const int to = __shfl_sync(0xffffffffu, out_row, r);
            const uint4 v = *reinterpret_cast<const uint4 *>(stage + r * 128 + ((p ^ (r & 7)) << 4));
            if (to >= 0) *reinterpret_cast<uint4 *>(out + (int64_t)to * ldo + n + p * 8) = v;
        }
        return;
    }
#pragma unroll 4
    for (int r = 0; r < 32; ++r) {
        const int to = __shfl_sync(0xffffffffu, out_row, r);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int e = h * 32 + lane;
            const __nv_bfloat16 v = *reinterpret_cast<const __nv_bfloat16 *>(stage + r * 128 + (((e >> 3) ^ (r & 7)) << 4) + (e & 7) * 2);
            if (to >= 0 && n + e < cols) out[(int64_t)to * ldo + n + e] = v;
        }
    }
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    const __nv_bfloat162 b2 = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&b2);
}
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// 32 values of a row, the half `h` of 64 columns, into the staging buffer; returns the sum of what was stored
__device__ __forceinline__ float stage32(unsigned char *stage, int lane, int h, const float *v)
{
    unsigned char *row = stage + lane * 128;
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w[e] = pack2(v[j * 8 + e * 2], v[j * 8 + e * 2 + 1]);
            s += low(w[e]) + high(w[e]);
        }
        *reinterpret_cast<uint4 *>(row + (((h * 4 + j) ^ (lane & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return s;
}

// f * W[k .. k + N, label] added to N neighbouring elements of a row of dH; VK: W is stored [V, K]
template <bool VK, int N>
__device__ __forceinline__ void add_label(const Args &a, float f, int label, int k, float *v)
{
    if (VK) {
        const __nv_bfloat16 *w = a.W + (int64_t)label * a.ldw + k;
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            if (k + j + 4 <= a.dim_n) {
                const uint2 x = __ldg(reinterpret_cast<const uint2 *>(w + j));
                v[j] = fmaf(f, low(x.x), v[j]);
                v[j + 1] = fmaf(f, high(x.x), v[j + 1]);
                v[j + 2] = fmaf(f, low(x.y), v[j + 2]);
                v[j + 3] = fmaf(f, high(x.y), v[j + 3]);
            } else {
#pragma unroll
                for (int e = j; e < j + 4; ++e)
                    if (k + e < a.dim_n) v[e] = fmaf(f, __bfloat162float(w[e]), v[e]);
            }
        }
    } else {
        const __nv_bfloat16 *w = a.W + (int64_t)k * a.ldw + label;
        float x[N];
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = k + j < a.dim_n ? __bfloat162float(w[(int64_t)j * a.ldw]) : 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = fmaf(f, x[j], v[j]);
    }
}

template <bool A_MN, bool B_MN, int PRODUCT>
__global__ void __launch_bounds__(kThreads, 1)
product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_a_all,
               const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_out, const Args a)
{
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ Smem sm;
    unsigned char *ring = smem_raw + ((1024u - (saddr(smem_raw) & 1023u)) & 1023u);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            barrier_init(&sm.full[s], 1);
            barrier_init(&sm.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            barrier_init(&sm.tmem_full[b], 1);
            barrier_init(&sm.tmem_empty[b], 2 * kEpiWarps);      // both blocks' epilogues
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) tmem_alloc_all_pair(&sm.tmem_base);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_barrier();                                          // the other block's barriers are ready too
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = sm.tmem_base;
    grid_dependents_may_launch();
    grid_dependency_wait();
    const int rank = (int)cluster_rank(), pair = blockIdx.x / 2, pairs = gridDim.x / 2;
    const int rows = rows_of(a);
    const Plan plan = plan_of<PRODUCT>(a, rows, pairs);
    Work work;
    work.init(plan, pair);

    if (warp == 0) {
        if (lane == 0) {
            // (all rows real: they have not been packed)
            const CUtensorMap *ma = PRODUCT == kLogits && *a.n_real == a.M ? &map_a_all : &map_a;
            const int row0 = PRODUCT == kLogits ? a.row0 : 0;
            bool alive = true;
            uint32_t it = 0, s = 0, parity = 1;                 // (waiting for the phase before the first returns at once)
            while (alive && work.next(plan, pairs)) {
                const int2 t = tile_of(work.u, plan.m_tiles, plan.n_tiles, a.gm, a.gn);
                const int m0 = t.x * kTile + rank * kBM, n0 = t.y * kTile + rank * kBM;
                for (int kb = work.kb0; kb < work.kb1; ++kb, ++it) {
                    wait_alive(alive, &sm.empty[s], parity, a.status);
                    if (!alive) break;
                    unsigned char *stage = ring + (size_t)s * kStage;
                    // (bytes of the other block may be counted before they are announced: the phase cannot end
                    // without the leader's arrival)
                    if (rank == 0) barrier_expect_tx(&sm.full[s], 2u * kStage);
                    const uint32_t bar = leader_addr(&sm.full[s]);
                    if (A_MN) {                                 // stored [k, m]: boxes of 64 (m) x 64 (k)
                        tma_load_2d_pair(stage, ma, m0, kb * kBlockK, bar);
                        tma_load_2d_pair(stage + kBox, ma, m0 + 64, kb * kBlockK, bar);
                    } else {                                    // stored [m, k]: one box of 64 (k) x 128 (m)
                        tma_load_2d_pair(stage, ma, kb * kBlockK, row0 + m0, bar);
                    }
                    if (B_MN) {
                        tma_load_2d_pair(stage + kHalf, &map_b, n0, kb * kBlockK, bar);
                        tma_load_2d_pair(stage + kHalf + kBox, &map_b, n0 + 64, kb * kBlockK, bar);
                    } else {
                        tma_load_2d_pair(stage + kHalf, &map_b, kb * kBlockK, n0, bar);
                    }
                    if (++s == kStages) { s = 0; parity ^= 1; }
                }
            }
            // copies in flight land before the block may end
            if (rank == 0)
                for (uint32_t i = it > kStages ? it - kStages : 0; i < it; ++i)
                    wait(&sm.full[i % kStages], (i / kStages) & 1, a.status);
            // and so do the last arrivals on this block's barriers, which no load waited for
            for (uint32_t i = it > kStages ? it - kStages : 0; i < it; ++i)
                wait_alive(alive, &sm.empty[i % kStages], (i / kStages) & 1, a.status);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0 && lane == 0) {
            constexpr uint32_t idesc = instr_desc(A_MN, B_MN, kTile, kTile);
            bool alive = true;
            uint32_t s = 0, s_parity = 0, tiles = 0;
            while (alive && work.next(plan, pairs)) {
                if (work.kb0 == work.kb1) continue;             // an empty contraction: the epilogue knows
                const uint32_t buf = tiles & 1;
                wait_alive(alive, &sm.tmem_empty[buf], ((tiles >> 1) & 1) ^ 1, a.status);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t tmem_d = tmem_base + buf * kTile;
                for (int kb = work.kb0; kb < work.kb1; ++kb) {
                    wait_alive(alive, &sm.full[s], s_parity, a.status);
                    if (!alive) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t a_addr = saddr(ring + (size_t)s * kStage), b_addr = a_addr + kHalf;
#pragma unroll
                    for (int kk = 0; kk < kBlockK / 16; ++kk) {
                        // K-major: 8-row groups 1024 bytes apart, 16 contraction elements are 32 bytes. MN-major: 64-wide
                        // boxes, 8 contraction rows 1024 bytes apart, 16 of them are 2048 bytes.
                        const uint64_t ad = A_MN ? smem_desc(a_addr + kk * 2048, kBox, 1024) : smem_desc(a_addr + kk * 32, 16, 1024);
                        const uint64_t bd = B_MN ? smem_desc(b_addr + kk * 2048, kBox, 1024) : smem_desc(b_addr + kk * 32, 16, 1024);
                        mma_pair(tmem_d, ad, bd, idesc, kb > work.kb0 || kk ? 1u : 0u);
                    }
                    commit_pair(&sm.empty[s]);
                    if (++s == kStages) { s = 0; s_parity ^= 1; }
                }
                if (alive && PPO_TEST_WITHHOLD_XENT != 1) {
                    commit_pair(&sm.tmem_full[buf]);
                    ++tiles;
                }
            }
            // every product has ended before tensor memory is freed
            for (uint32_t i = tiles > 2 ? tiles - 2 : 0; i < tiles; ++i) wait(&sm.tmem_full[i & 1], (i >> 1) & 1, a.status);
            // and the other block's last arrivals before this block ends
            for (uint32_t i = tiles > 2 ? tiles - 2 : 0; i < tiles; ++i)
                wait_alive(alive, &sm.tmem_empty[i & 1], (i >> 1) & 1, a.status);
        }
        __syncwarp();
    } else if (warp >= 4) {
        const int q = warp & 3, h = (warp - 4) >> 2;            // lanes 32 q .., columns 128 h .. of the tile
        unsigned char *const stages = ring + (size_t)kStages * kStage + (warp - 4) * 2 * kStageOut;
        unsigned char *stage = stages;
        const uint32_t tmem_empty = leader_addr(&sm.tmem_empty[0]);
        const float nan = __int_as_float(0x7fffffff);
        bool alive = true;
        uint32_t tiles = 0;
        while (work.next(plan, pairs)) {
            const int2 t = tile_of(work.u, plan.m_tiles, plan.n_tiles, a.gm, a.gn);
            const int m_warp = t.x * kTile + rank * kBM + q * 32, n = t.y * kTile + h * 128;
            const int row = m_warp + lane;
            const bool empty = work.kb0 == work.kb1;
            const uint32_t buf = tiles & 1;
            const uint32_t taddr = tmem_base + buf * kTile + h * 128 + ((uint32_t)(q * 32) << 16);
            bool ok = false;
            int label = -1, out_row = -1;
            float base = 0.f;
            float2 scale = make_float2(0.f, 0.f);
            if (PRODUCT == kLogits) {
                ok = row < rows;
                if (ok) {
                    label = a.labels[a.order[a.row0 + row]] - n;
                    base = a.base[a.row0 + row];
                }
            } else if (PRODUCT == kHidden) {
                ok = row < rows;
                if (ok && work.part < 0) {
                    out_row = a.order[a.row0 + row];
                    scale = a.row_scale[row];
                    label = scale.y != 0.f ? a.labels[out_row] : -1;
                }
            } else {
                ok = row < a.dim_m;
                out_row = ok ? row : -1;
            }
            if (!empty) {
                wait_alive(alive, &sm.tmem_full[buf], (tiles >> 1) & 1, a.status);
                alive = __all_sync(0xffffffffu, alive);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            }
            // this warp's read of 32 columns; after the tile's last one the accumulator is released
            const auto read = [&](int cc, bool last, float *v) {
                if (empty) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = 0.f;
                    return;
                }
                uint32_t r[32];
                __syncwarp();
                tmem_ld32(taddr + cc * 32, r);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                if (last) {
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    barrier_arrive_cluster_if(tmem_empty + buf * 8, lane == 0 && alive && PPO_TEST_WITHHOLD_XENT != 2);
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = alive ? __uint_as_float(r[j]) : nan;
            };
            // 64 columns of the staging buffer, from column c64 of the warp's half
            const auto send = [&](int c64, bool bulk) {
                if (bulk) {
                    fence_async_proxy();
                    __syncwarp();
                    if (lane == 0) tma_store_2d(&map_out, n + c64, m_warp, stage);
                } else {
                    __syncwarp();
                    store_rows(stage, a.out, a.ldo, out_row, n + c64, a.dim_n);
                    __syncwarp();
                }
            };
            // the other staging buffer, whose last copy has read it
            const auto reuse = [&] {
                stage = stage == stages ? stages + kStageOut : stages;
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                __syncwarp();
            };

            if (PRODUCT == kLogits) {
                float m = kNoRef;
#pragma unroll 1
                for (int cc = 0; cc < 4; ++cc) {
                    float v[32];
                    read(cc, false, v);
                    const int left = a.dim_n - n - cc * 32;
                    if (left >= 32) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) m = fmaxf(m, v[j]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) m = j < left ? fmaxf(m, v[j]) : m;
                    }
                }
                const float ref = base + 128.f * rintf((fmaxf(m * a.c, -1e9f) - base) * (1.f / 128.f));
                float s = 0.f, rounded = 0.f;
#pragma unroll 1
                for (int cc = 0; cc < 4; ++cc) {
                    float v[32];
                    read(cc, cc == 3, v);
                    if ((unsigned)(label - cc * 32) < 32u) {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (label - cc * 32 == j) a.picked[row] = v[j];
                    }
                    const int left = ok ? a.dim_n - n - cc * 32 : 0;
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const float e = ex2(fmaf(v[j], a.c, -ref));
                        v[j] = j < left ? e : 0.f;
                        s += v[j];
                    }
                    if (a.store) {
                        if ((cc & 1) == 0) reuse();
                        rounded += stage32(stage, lane, cc & 1, v);
                        if ((cc & 1) && n + (cc - 1) * 32 < a.dim_n) send((cc - 1) * 32, true);
                    }
                }
                if (ok && n < a.dim_n) a.part[(size_t)row * a.chunks + n / kChunk] = make_float4(ref, s, rounded, 0.f);
            } else if (PRODUCT == kHidden) {
                // (four columns of 256 rows follow one another in scratch: a warp writes 512 bytes at a time)
                float4 *part = reinterpret_cast<float4 *>(a.scratch + (size_t)(pair * 2 + max(work.part, 0)) * kTileFloats) +
                               h * 32 * kTile + rank * kBM + q * 32 + lane;
#pragma unroll 1
                for (int cc = 0; cc < 4; ++cc) {
                    float v[32];
                    read(cc, cc == 3, v);
                    if (work.part >= 0) {
                        if (!ok) continue;
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            part[(cc * 8 + j) * kTile] = make_float4(v[j * 4], v[j * 4 + 1], v[j * 4 + 2], v[j * 4 + 3]);
                        continue;
                    }
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] *= scale.x;
                    if (label >= 0) add_label<B_MN, 32>(a, scale.y, label, n + cc * 32, v);
                    stage32(stage, lane, cc & 1, v);
                    if ((cc & 1) && n + (cc - 1) * 32 < a.dim_n) send((cc - 1) * 32, false);
                }
            } else {
                const bool first = a.row0 == 0, last = a.row0 + a.rows_max >= *a.n_real;
                float4 *sum = reinterpret_cast<float4 *>(a.scratch + ((size_t)t.x * plan.n_tiles + t.y) * kTileFloats) +
                              h * 32 * kTile + rank * kBM + q * 32 + lane;
#pragma unroll 1
                for (int cc = 0; cc < 4; ++cc) {
                    float4 old[8];
                    if (!first) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) old[j] = sum[(cc * 8 + j) * kTile];
                    }
                    float v[32];
                    read(cc, cc == 3, v);
                    if (!first) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            v[j * 4] += old[j].x; v[j * 4 + 1] += old[j].y; v[j * 4 + 2] += old[j].z; v[j * 4 + 3] += old[j].w;
                        }
                    }
                    if (!last) {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            sum[(cc * 8 + j) * kTile] = make_float4(v[j * 4], v[j * 4 + 1], v[j * 4 + 2], v[j * 4 + 3]);
                        continue;
                    }
                    if ((cc & 1) == 0) reuse();
                    stage32(stage, lane, cc & 1, v);
                    const int col = n + (cc - 1) * 32;
                    if ((cc & 1) && col < a.dim_n) {
                        const bool bulk = col + 64 <= a.bulk_cols;
                        if (!bulk || m_warp < a.dim_m) send((cc - 1) * 32, bulk);
                    }
                }
            }
            if (!empty) ++tiles;
        }
        if (lane == 0) tma_store_wait_read();                   // shared memory outlives the copies out of it
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_barrier();                                          // neither block ends while the other may reach into it
    if (warp == 0) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        tmem_free_all_pair(tmem_base);
    }
}

// The tiles of dH that were cut along the vocabulary: a block adds up 32 rows x 64 columns over the pairs that hold parts of
// them, in the order of the contraction, and turns them in shared memory so that rows leave in runs.
constexpr int kJoinThreads = 256, kJoinBlocks = (kTile / 32) * (kTile / 64);
template <bool VK>
__global__ void __launch_bounds__(kJoinThreads)
join_kernel(const Args a, int pairs)
{
    __shared__ float4 turn[32][17];
    grid_dependents_may_launch();
    grid_dependency_wait();
    const int rows = rows_of(a);
    const Plan p = plan_of<kHidden>(a, rows, pairs);
    const int rest = blockIdx.x / kJoinBlocks, part_of = blockIdx.x % kJoinBlocks;
    if (rest >= p.n_rest) return;
    const int row0 = (part_of % (kTile / 32)) * 32, j0 = part_of / (kTile / 32) * 16;
    const int2 t = tile_of(p.n_whole + rest, p.m_tiles, p.n_tiles, a.gm, a.gn);
    const int m0 = t.x * kTile + row0, n0 = t.y * kTile + j0 * 4;
    if (m0 >= rows || n0 >= a.dim_n) return;
    const int first = (int)((int64_t)rest * p.kbs / p.share), last = (int)(((int64_t)(rest + 1) * p.kbs - 1) / p.share);
    const int lane = threadIdx.x & 31, jj = threadIdx.x >> 5;
    float4 v[2];
    v[0] = v[1] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int c = first; c <= last; ++c) {
        const int part = rest - (int)((int64_t)c * p.share / p.kbs);     // the pair's first or second tile
        const float4 *from = reinterpret_cast<const float4 *>(a.scratch + (size_t)(c * 2 + part) * kTileFloats) + row0 + lane;
        const float4 x = from[(j0 + jj) * kTile], y = from[(j0 + jj + 8) * kTile];
        v[0].x += x.x; v[0].y += x.y; v[0].z += x.z; v[0].w += x.w;
        v[1].x += y.x; v[1].y += y.y; v[1].z += y.z; v[1].w += y.w;
    }
    turn[lane][jj] = v[0];
    turn[lane][jj + 8] = v[1];
    __syncthreads();
    const int c4 = threadIdx.x & 15;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = (threadIdx.x >> 4) + h * 16, n = n0 + c4 * 4;
        if (m0 + r >= rows || n >= a.dim_n) continue;
        const float2 s = a.row_scale[m0 + r];
        const float4 x = turn[r][c4];
        float y[4] = {x.x * s.x, x.y * s.x, x.z * s.x, x.w * s.x};
        const int row = a.order[a.row0 + m0 + r];
        if (s.y != 0.f) add_label<VK, 4>(a, s.y, a.labels[row], n, y);
        __nv_bfloat16 *to = a.out + (int64_t)row * a.ldo + n;
        if (n + 4 <= a.dim_n && reinterpret_cast<uintptr_t>(to) % 8 == 0) {
            *reinterpret_cast<uint2 *>(to) = make_uint2(pack2(y[0], y[1]), pack2(y[2], y[3]));
        } else {
            for (int e = 0; e < 4 && n + e < a.dim_n; ++e) to[e] = __float2bfloat16_rn(y[e]);
        }
    }
}

// ---------------------------------------------------------------- rows
struct RowArgs {
    const __nv_bfloat16 *H;
    int64_t ldh, lddh;
    int M, K, V, Kp;                                            // Kp: row pitch of the packed and the scaled rows
    const int32_t *labels;
    const uint8_t *mask;
    int32_t ignore_id;
    float c, inv_tau, scale;
    const float *denom;
    int32_t *order;                                             // [M] real rows, ascending; then the others
    int *n_real;
    const __nv_bfloat16 *W;
    int64_t ldw;
    int vk;
    float *w_mean;                                              // [K] mean of kSample columns of W
    float *base;                                                // [M] reference of real row i
    __nv_bfloat16 *packed;                                      // [M, Kp] (written when some row is left out)
    __nv_bfloat16 *scaled;                                      // [rows_max, Kp] a H; null: no gradients
    __nv_bfloat16 *u;                                           // [rows_max, Vp]
    int64_t Vp;
    float *picked;
    float2 *row_scale;
    float4 *part;
    int chunks, row0, rows_max;
    float *loss, *nll, *lse;
    __nv_bfloat16 *dH;
    int *status;
};

// The mean of kSample neighbouring columns of W, from the middle of the vocabulary, for 128 hidden elements: a thread loads
// eight neighbours in memory, eight (stored [K, V]) or 64 (stored [V, K]) threads share an element. (One element after the
// other, 64 loads each: 36 us at K = 4096, most of it misses of the address translation.)
constexpr int kOrderThreads = 1024, kOrderPer = 8, kSample = 64, kMeanPer = kOrderThreads / 8;
__device__ __forceinline__ void mean_columns(const RowArgs &a, int k0, float (*part)[kMeanPer])
{
    const int v0 = min(a.V / 2, max(0, a.V - kSample)) & ~7, n = min(kSample, a.V - v0);
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (a.vk) {
        // four times 16 rows of W
        const int k = k0 + (threadIdx.x & 15) * 8;
#pragma unroll
        for (int j = threadIdx.x >> 4; j < kSample; j += kOrderThreads / 16) {
            if (j >= n) break;
            const __nv_bfloat16 *w = a.W + (int64_t)(v0 + j) * a.ldw + k;
            if (k + 8 <= a.K) {
                const uint4 y = *reinterpret_cast<const uint4 *>(w);
                const uint32_t z[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] += e & 1 ? high(z[e / 2]) : low(z[e / 2]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (k + e < a.K) x[e] += __bfloat162float(w[e]);
            }
        }
        // lanes 16 apart hold other rows for the same elements; then the warps
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += __shfl_xor_sync(0xffffffffu, x[e], 16);
        if ((threadIdx.x & 31) < 16)
#pragma unroll
            for (int e = 0; e < 8; ++e) part[threadIdx.x >> 5][(threadIdx.x & 15) * 8 + e] = x[e];
        __syncthreads();
        if (threadIdx.x < kMeanPer && k0 + (int)threadIdx.x < a.K) {
            float s = 0.f;
            for (int w = 0; w < kOrderThreads / 32; ++w) s += part[w][threadIdx.x];
            a.w_mean[k0 + threadIdx.x] = s / (float)n;
        }
        return;
    }
    const int k = k0 + (threadIdx.x >> 3), v = v0 + (threadIdx.x & 7) * 8;
    float s = 0.f;
    if (k < a.K) {
        const __nv_bfloat16 *w = a.W + (int64_t)k * a.ldw + v;
        if (v + 8 <= a.V) {
            const uint4 y = *reinterpret_cast<const uint4 *>(w);
            s = low(y.x) + high(y.x) + low(y.y) + high(y.y) + low(y.z) + high(y.z) + low(y.w) + high(y.w);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (v + e < a.V) s += __bfloat162float(w[e]);
        }
    }
#pragma unroll
    for (int off = 1; off < 8; off <<= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    if (k < a.K && (threadIdx.x & 7) == 0) a.w_mean[k] = s / (float)n;
}

// Block 0: the real rows' order. The others: mean_columns.
__global__ void __launch_bounds__(kOrderThreads)
order_kernel(const RowArgs a)
{
    grid_dependents_may_launch();
    __shared__ float part[kOrderThreads / 32][kMeanPer];
    if (blockIdx.x > 0) {
        mean_columns(a, (blockIdx.x - 1) * kMeanPer, part);
        return;
    }
    __shared__ int warp_sum[32], carry;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) carry = 0;
    __syncthreads();
    const bool wide = reinterpret_cast<uintptr_t>(a.labels) % 16 == 0 && reinterpret_cast<uintptr_t>(a.mask) % 8 == 0;
    for (int64_t base = 0; base < a.M; base += kOrderThreads * kOrderPer) {
        const int64_t i0 = base + threadIdx.x * kOrderPer;
        unsigned bits = 0;
        if (wide && i0 + kOrderPer <= a.M) {
            const int4 x = reinterpret_cast<const int4 *>(a.labels + i0)[0], y = reinterpret_cast<const int4 *>(a.labels + i0)[1];
            const uint2 m = a.mask ? *reinterpret_cast<const uint2 *>(a.mask + i0) : make_uint2(~0u, ~0u);
            const int l[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (((e < 4 ? m.x : m.y) >> (8 * (e & 3)) & 255) && l[e] != a.ignore_id) bits |= 1u << e;
        } else {
#pragma unroll
            for (int e = 0; e < kOrderPer; ++e)
                if (i0 + e < a.M && (!a.mask || a.mask[i0 + e]) && a.labels[i0 + e] != a.ignore_id) bits |= 1u << e;
        }
        const int mine = __popc(bits);
        int incl = mine;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += o;
        }
        if (lane == 31) warp_sum[warp] = incl;
        __syncthreads();
        const int w = warp_sum[lane];
        int at = carry + __reduce_add_sync(0xffffffffu, lane < warp ? w : 0) + incl - mine;
#pragma unroll
        for (int e = 0; e < kOrderPer; ++e) {
            if (i0 + e >= a.M) break;
            // (the rows left out fill the array from its end)
            if (bits >> e & 1) a.order[at++] = (int)(i0 + e);
            else a.order[a.M - 1 - (int)(i0 + e - at)] = (int)(i0 + e);
        }
        __syncthreads();
        if (threadIdx.x == kOrderThreads - 1) carry = at;
        __syncthreads();
    }
    if (threadIdx.x == 0) *a.n_real = carry;
}

constexpr int kRowThreads = 256;
// real rows: their reference, and a packed copy where some rows are left out; those get their zeros
__global__ void __launch_bounds__(kRowThreads)
pack_kernel(const RowArgs a)
{
    __shared__ float red[kRowThreads / 32];
    grid_dependents_may_launch();
    grid_dependency_wait();
    const int n = *a.n_real, i = blockIdx.x;
    const int row = a.order[i];
    if (i >= n) {
        if (threadIdx.x == 0) {
            a.nll[row] = 0.f;
            if (a.lse) a.lse[row] = 0.f;
        }
        if (a.dH)
            for (int k = threadIdx.x; k < a.K; k += kRowThreads) a.dH[(int64_t)row * a.lddh + k] = __float2bfloat16_rn(0.f);
        return;
    }
    const __nv_bfloat16 *from = a.H + (int64_t)row * a.ldh;
    __nv_bfloat16 *to = a.packed + (int64_t)i * a.Kp;
    float s = 0.f;
    for (int k = threadIdx.x * 8; k < a.K; k += kRowThreads * 8) {
        if (k + 8 <= a.K) {
            const uint4 v = *reinterpret_cast<const uint4 *>(from + k);
            if (n < a.M) *reinterpret_cast<uint4 *>(to + k) = v;
            const float4 p = *reinterpret_cast<const float4 *>(a.w_mean + k), q = *reinterpret_cast<const float4 *>(a.w_mean + k + 4);
            s = fmaf(low(v.x), p.x, s); s = fmaf(high(v.x), p.y, s); s = fmaf(low(v.y), p.z, s); s = fmaf(high(v.y), p.w, s);
            s = fmaf(low(v.z), q.x, s); s = fmaf(high(v.z), q.y, s); s = fmaf(low(v.w), q.z, s); s = fmaf(high(v.w), q.w, s);
        } else {
            for (int e = k; e < a.K; ++e) {
                if (n < a.M) to[e] = from[e];
                s = fmaf(__bfloat162float(from[e]), a.w_mean[e], s);
            }
        }
    }
    s = warp_sum_f(s);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.f;
#pragma unroll
        for (int w = 0; w < kRowThreads / 32; ++w) s += red[w];
        // the middle of the window; whole numbers, so that y - reference loses nothing that y does not
        s = rintf(s * a.c) + 32.f;
        a.base[i] = fabsf(s) < 1e9f ? s : 0.f;
    }
}

// A row's statistics out of its chunks', its loss and the factors of its gradient; U at the label; a H
__global__ void __launch_bounds__(kRowThreads)
row_kernel(const RowArgs a)
{
    __shared__ float red[3][kRowThreads / 32];
    grid_dependents_may_launch();
    grid_dependency_wait();
    const int n_real = *a.n_real, rows = max(0, min(a.rows_max, n_real - a.row0)), r = blockIdx.x;
    __nv_bfloat16 *scaled = a.scaled ? a.scaled + (int64_t)r * a.Kp : nullptr;
    if (r >= rows) {
        // up to the next block of the contraction: zeros that product 3 reads (U has its own)
        if (scaled && r < (rows + kBlockK - 1) / kBlockK * kBlockK)
            for (int k = threadIdx.x; k < a.K; k += kRowThreads) scaled[k] = __float2bfloat16_rn(0.f);
        return;
    }
    const int row = a.order[a.row0 + r], lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int label = a.labels[row];
    const bool bad = label < 0 || label >= a.V;
    const float4 *part = a.part + (size_t)r * a.chunks;
    float m = kNoRef;
    for (int t = threadIdx.x; t < a.chunks; t += kRowThreads) m = fmaxf(m, part[t].x);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
    if (lane == 0) red[0][warp] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kRowThreads / 32; ++w) m = fmaxf(m, red[0][w]);
    float s = 0.f, sr = 0.f;                                    // sums of U and of the rounded U
    for (int t = threadIdx.x; t < a.chunks; t += kRowThreads) {
        const float4 p = part[t];
        const float f = ex2(p.x - m);
        s = fmaf(p.y, f, s);
        sr = fmaf(p.z, f, sr);
        if (p.x != m && a.u) {
            // (16-byte pieces of 8 columns; the columns behind V are not used)
            uint4 *u = reinterpret_cast<uint4 *>(a.u + (int64_t)r * a.Vp + (int64_t)t * kChunk);
            const int64_t left = a.Vp - (int64_t)t * kChunk;
            for (int j = 0; j < kChunk / 8 && j * 8 < left; ++j) {
                uint4 v = u[j];
                uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = pack2(low(w[e]) * f, high(w[e]) * f);
                u[j] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
    s = warp_sum_f(s);
    sr = warp_sum_f(sr);
    if (lane == 0) {
        red[1][warp] = s;
        red[2][warp] = sr;
    }
    __syncthreads();
    s = sr = 0.f;
#pragma unroll
    for (int w = 0; w < kRowThreads / 32; ++w) {
        s += red[1][w];
        sr += red[2][w];
    }
    const float l2s = log2f(s), nan = __int_as_float(0x7fffffff);
    const float acc = bad ? nan : a.picked[r];
    if (threadIdx.x == 0) {
        a.nll[row] = ((m - acc * a.c) + l2s) * kLn2;
        if (a.lse) a.lse[row] = (m + l2s) * kLn2;
        if (bad && a.status) atomicOr(a.status, PPO_DEV_BAD_TOKEN);
    }
    if (!a.u) return;
    // U at the label, as product 1 stored it, less S; in bf16, and what that leaves
    float f2 = nan, f3 = nan, left = 0.f;
    if (!bad) {
        const float ref = part[label / kChunk].x;
        const float u = __bfloat162float(__float2bfloat16_rn(ex2(fmaf(acc, a.c, -ref)))) * ex2(ref - m);
        const float want = u - sr;
        const __nv_bfloat16 stored = __float2bfloat16_rn(want);
        const float got = __bfloat162float(stored);
        f2 = a.scale * a.inv_tau / ((a.denom ? *a.denom : (float)n_real) * sr);
        f3 = got != 0.f ? f2 * (want / got) : f2;
        left = f2 * (want - got);
        if (threadIdx.x == 0) a.u[(int64_t)r * a.Vp + label] = stored;
    }
    if (threadIdx.x == 0) a.row_scale[r] = make_float2(f2, left);
    if (!scaled) return;
    const __nv_bfloat16 *h = a.H + (int64_t)row * a.ldh;
    for (int k = threadIdx.x * 8; k < a.K; k += kRowThreads * 8) {
        if (k + 8 <= a.K) {
            const uint4 v = *reinterpret_cast<const uint4 *>(h + k);
            uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = pack2(low(w[e]) * f3, high(w[e]) * f3);
            *reinterpret_cast<uint4 *>(scaled + k) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            for (int e = k; e < a.K; ++e) scaled[e] = __float2bfloat16_rn(__bfloat162float(h[e]) * f3);
        }
    }
}

constexpr int kLossThreads = 1024;
__global__ void __launch_bounds__(kLossThreads)
loss_kernel(const RowArgs a)
{
    __shared__ double red[32];
    grid_dependency_wait();
    double s = 0.0;
#pragma unroll 4
    for (int i = threadIdx.x; i < a.M; i += kLossThreads) s += (double)a.nll[i];
    s = block_sum<kLossThreads>(s, red);
    if (threadIdx.x == 0) {
        const int n = *a.n_real;
        *a.loss = n ? (float)(s / (a.denom ? (double)*a.denom : (double)n)) : 0.f;
        if (!n && a.status) atomicOr(a.status, PPO_DEV_EMPTY_MASK);
    }
}

// ---------------------------------------------------------------- host side
struct Layout {
    int pieces, rows_max, chunks, Kp;
    int64_t Vp;
    size_t n_real, order, base, w_mean, picked, row_scale, part, packed, scaled, u, parts, sums, bytes;
};

// Pieces of at most 8192 rows by default: at V = 50304 that is 824 MB of U, and the sums of dW, read and written once a
// piece, are under a tenth of the piece's traffic.
static Layout layout_of(int64_t M, int64_t K, int64_t V, int64_t piece_rows, bool dh, bool dw)
{
    Layout l;
    const int64_t most = piece_rows > 0 ? piece_rows : 8192;
    l.pieces = (int)((M + most - 1) / most);
    const int64_t even = (M + l.pieces - 1) / l.pieces;
    l.rows_max = (int)((even + kTile - 1) / kTile * kTile);
    l.pieces = (int)((M + l.rows_max - 1) / l.rows_max);
    l.chunks = (int)((V + kChunk - 1) / kChunk);
    l.Kp = (int)((K + 7) / 8 * 8);
    l.Vp = (V + 7) / 8 * 8;
    size_t at = 0;
    const auto take = [&](size_t n) {
        const size_t here = at;
        at += align256(n);
        return here;
    };
    const bool grad = dh || dw;
    const size_t rows = (size_t)l.rows_max;
    l.n_real = take(4);
    l.order = take((size_t)M * 4);
    l.base = take((size_t)M * 4);
    l.w_mean = take((size_t)K * 4);
    l.picked = take(rows * 4);
    l.row_scale = take(rows * sizeof(float2));
    l.part = take(rows * (size_t)l.chunks * sizeof(float4));
    l.packed = take((size_t)M * l.Kp * 2);
    l.scaled = take(dw ? rows * l.Kp * 2 : 0);
    l.u = take(grad ? rows * (size_t)l.Vp * 2 : 0);
    l.parts = take(dh ? (size_t)kMaxPairs * 2 * kTileFloats * 4 : 0);
    const size_t tiles = (size_t)((K + kTile - 1) / kTile) * (size_t)((V + kTile - 1) / kTile);
    l.sums = take(dw && l.pieces > 1 ? tiles * kTileFloats * 4 : 0);
    l.bytes = at;
    return l;
}

static int pairs_of_device(int *pairs)
{
    int dev = 0, sms = 148;
    PPO_RETURN_IF_CUDA(cudaGetDevice(&dev));
    PPO_RETURN_IF_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    *pairs = sms / 2 < kMaxPairs ? sms / 2 : kMaxPairs;
    return PPO_OK;
}

template <bool A_MN, bool B_MN, int PRODUCT>
static int launch_product(const CUtensorMap &ma, const CUtensorMap &ma_all, const CUtensorMap &mb, const CUtensorMap &mo, Args a,
                          int pairs, cudaStream_t s)
{
    auto kern = product_kernel<A_MN, B_MN, PRODUCT>;
    PPO_RETURN_IF_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * pairs));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cudaError_t e = cudaLaunchKernelEx(&cfg, kern, ma, ma_all, mb, mo, a);
    if (e != cudaSuccess) {   // attribute not accepted in this context: ordinary launch (same results, no overlap)
        (void)cudaGetLastError();
        cfg.numAttrs = 1;
        e = cudaLaunchKernelEx(&cfg, kern, ma, ma_all, mb, mo, a);
    }
    PPO_RETURN_IF_CUDA(e);
    return PPO_OK;
}

constexpr int64_t kLimit = ((int64_t)1 << 31) - 16384;

static bool sizes_ok(int64_t M, int64_t K, int64_t V, int64_t piece_rows)
{
    return M > 0 && K > 0 && V > 0 && M < kLimit && K < kLimit && V < kLimit && piece_rows >= 0 &&
           ((K + 255) / 256) * ((V + 255) / 256) < ((int64_t)1 << 30) && ((M + 255) / 256) * ((V + 255) / 256) < ((int64_t)1 << 30);
}

}   // namespace xent
}   // namespace ppo

using namespace ppo;

extern "C" size_t ppo_lmhead_xent_scratch_bytes(int64_t M, int64_t K, int64_t V, int64_t piece_rows, int want_dh, int want_dw)
{
    return xent::sizes_ok(M, K, V, piece_rows) ? xent::layout_of(M, K, V, piece_rows, want_dh != 0, want_dw != 0).bytes : 0;
}

extern "C" int ppo_lmhead_xent(const void *H, int64_t ldh, const void *W, int64_t ldw, int w_layout, int64_t M, int64_t K, int64_t V,
                               const int32_t *labels, const uint8_t *mask, int32_t ignore_id, float temperature, float scale,
                               const float *denom, int64_t piece_rows, float *loss, float *nll, float *lse, void *dH, int64_t lddh,
                               void *dW, int64_t lddw, void *workspace, void *scratch, void *stream)
{
    using namespace xent;
    if (w_layout != PPO_W_KV && w_layout != PPO_W_VK) return PPO_ERR_PARAM;
    const bool vk = w_layout == PPO_W_VK;
    const int64_t w_inner = vk ? K : V, w_outer = vk ? V : K;
    if (!sizes_ok(M > 0 ? M : 1, K, V, piece_rows) || M < 0 || ldh < K || ldw < w_inner || (dH && lddh < K) || (dW && lddw < w_inner))
        return PPO_ERR_SHAPE;
    if (!(temperature > 0.f) || !finite_f(temperature) || !finite_f(scale)) return PPO_ERR_PARAM;
    if (!loss || !W) return PPO_ERR_NULL;
    if (M > 0 && (!H || !labels || !nll || !scratch)) return PPO_ERR_NULL;
    if (ldh % 8 || ldw % 8) return PPO_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(H) % 16 || reinterpret_cast<uintptr_t>(W) % 16 || reinterpret_cast<uintptr_t>(scratch) % 256 ||
        reinterpret_cast<uintptr_t>(dH) % 2 || reinterpret_cast<uintptr_t>(dW) % 2 || reinterpret_cast<uintptr_t>(labels) % 4)
        return PPO_ERR_ALIGN;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    int *status = workspace ? &ws_header(workspace)->status : nullptr;
    if (M == 0) {
        PPO_RETURN_IF_CUDA(cudaMemsetAsync(loss, 0, 4, s));
        if (dW) PPO_RETURN_IF_CUDA(cudaMemset2DAsync(dW, (size_t)lddw * 2, 0, (size_t)w_inner * 2, (size_t)w_outer, s));
        return PPO_OK;
    }
    int pairs = 0;
    int rc = pairs_of_device(&pairs);
    if (rc) return rc;
    const Layout l = layout_of(M, K, V, piece_rows, dH != nullptr, dW != nullptr);
    unsigned char *mem = reinterpret_cast<unsigned char *>(scratch);
    const bool grad = dH || dW;

    RowArgs r = {};
    r.H = reinterpret_cast<const __nv_bfloat16 *>(H);
    r.ldh = ldh; r.lddh = lddh; r.M = (int)M; r.K = (int)K; r.V = (int)V; r.Kp = l.Kp;
    r.labels = labels; r.mask = mask; r.ignore_id = ignore_id;
    r.c = kLog2e / temperature; r.inv_tau = 1.f / temperature; r.scale = scale; r.denom = denom;
    r.n_real = reinterpret_cast<int *>(mem + l.n_real);
    r.order = reinterpret_cast<int32_t *>(mem + l.order);
    r.W = reinterpret_cast<const __nv_bfloat16 *>(W); r.ldw = ldw; r.vk = vk;
    r.w_mean = reinterpret_cast<float *>(mem + l.w_mean);
    r.base = reinterpret_cast<float *>(mem + l.base);
    r.packed = reinterpret_cast<__nv_bfloat16 *>(mem + l.packed);
    r.scaled = dW ? reinterpret_cast<__nv_bfloat16 *>(mem + l.scaled) : nullptr;
    r.u = grad ? reinterpret_cast<__nv_bfloat16 *>(mem + l.u) : nullptr;
    r.Vp = l.Vp;
    r.picked = reinterpret_cast<float *>(mem + l.picked);
    r.row_scale = reinterpret_cast<float2 *>(mem + l.row_scale);
    r.part = reinterpret_cast<float4 *>(mem + l.part);
    r.chunks = l.chunks; r.rows_max = l.rows_max;
    r.loss = loss; r.nll = nll; r.lse = lse; r.dH = reinterpret_cast<__nv_bfloat16 *>(dH);
    r.status = status;

    CUtensorMap m_packed, m_h, m_w1, m_w2, m_u1, m_u2, m_u3, m_scaled, m_dw = {};
    if ((rc = make_map_pitch(&m_packed, r.packed, (uint64_t)K, (uint64_t)M, (uint64_t)l.Kp, kBM))) return rc;
    if ((rc = make_map_pitch(&m_h, H, (uint64_t)K, (uint64_t)M, (uint64_t)ldh, kBM))) return rc;
    // product 1 takes W with the vocabulary as the result's columns, product 2 with the hidden size
    if ((rc = make_map_pitch(&m_w1, W, (uint64_t)w_inner, (uint64_t)w_outer, (uint64_t)ldw, vk ? kBM : 64))) return rc;
    if ((rc = make_map_pitch(&m_w2, W, (uint64_t)w_inner, (uint64_t)w_outer, (uint64_t)ldw, vk ? 64 : kBM))) return rc;
    if (grad) {
        if ((rc = make_map_pitch(&m_u1, r.u, (uint64_t)V, (uint64_t)l.rows_max, (uint64_t)l.Vp, 32))) return rc;   // stores
        if ((rc = make_map_pitch(&m_u2, r.u, (uint64_t)V, (uint64_t)l.rows_max, (uint64_t)l.Vp, kBM))) return rc;
        if ((rc = make_map_pitch(&m_u3, r.u, (uint64_t)V, (uint64_t)l.rows_max, (uint64_t)l.Vp, 64))) return rc;
    } else {
        m_u1 = m_h;
    }

    Args a = {};
    a.n_real = r.n_real; a.M = (int)M; a.rows_max = l.rows_max; a.status = status;
    a.c = r.c; a.labels = labels; a.order = r.order; a.base = r.base; a.picked = r.picked; a.part = r.part; a.chunks = l.chunks; a.store = grad;
    a.row_scale = r.row_scale;
    Args a1 = a, a2 = a, a3 = a;
    a1.dim_m = l.rows_max; a1.dim_n = (int)V; a1.dim_k = (int)K; a1.gm = 9; a1.gn = 8;
    a2.dim_m = l.rows_max; a2.dim_n = (int)K; a2.dim_k = (int)V; a2.gm = 9; a2.gn = 8;
    a2.out = r.dH; a2.ldo = lddh; a2.W = reinterpret_cast<const __nv_bfloat16 *>(W); a2.ldw = ldw;
    a2.scratch = reinterpret_cast<float *>(mem + l.parts);
    a3.dim_m = (int)w_outer; a3.dim_n = (int)w_inner; a3.dim_k = l.rows_max; a3.gm = 8; a3.gn = 9;
    a3.out = reinterpret_cast<__nv_bfloat16 *>(dW); a3.ldo = lddw;
    a3.scratch = reinterpret_cast<float *>(mem + l.sums);
    if (dW) {
        if ((rc = make_map_pitch(&m_scaled, r.scaled, (uint64_t)K, (uint64_t)l.rows_max, (uint64_t)l.Kp, 64))) return rc;
        if (reinterpret_cast<uintptr_t>(dW) % 16 == 0 && lddw % 8 == 0 && lddw < ((int64_t)1 << 38)) {
            // (a box is clipped in units of 16 bytes: it would write zeros behind a row whose end is none)
            a3.bulk_cols = w_inner % 8 ? (int)w_inner : 0x7fffffff;
            if ((rc = make_map_pitch(&m_dw, dW, (uint64_t)w_inner, (uint64_t)w_outer, (uint64_t)lddw, 32))) return rc;
        }
    }

    // (the first launch waits for all work before the call, the others for the one before them)
    order_kernel<<<1 + (unsigned)((K + kMeanPer - 1) / kMeanPer), kOrderThreads, 0, s>>>(r);
    if ((rc = launch_status())) return rc;
    PPO_RETURN_IF_CUDA(launch_dependent(pack_kernel, dim3((unsigned)M), dim3(kRowThreads), 0, s, r));
    for (int p = 0; p < l.pieces; ++p) {
        r.row0 = a1.row0 = a2.row0 = a3.row0 = p * l.rows_max;
        rc = vk ? launch_product<false, false, kLogits>(m_packed, m_h, m_w1, m_u1, a1, pairs, s)
                : launch_product<false, true, kLogits>(m_packed, m_h, m_w1, m_u1, a1, pairs, s);
        if (rc) return rc;
        PPO_RETURN_IF_CUDA(launch_dependent(row_kernel, dim3((unsigned)l.rows_max), dim3(kRowThreads), 0, s, r));
        if (dH) {
            rc = vk ? launch_product<false, true, kHidden>(m_u2, m_u2, m_w2, m_u2, a2, pairs, s)
                    : launch_product<false, false, kHidden>(m_u2, m_u2, m_w2, m_u2, a2, pairs, s);
            if (rc) return rc;
            PPO_RETURN_IF_CUDA(launch_dependent(vk ? join_kernel<true> : join_kernel<false>, dim3((unsigned)((pairs - 1) * kJoinBlocks)),
                                                dim3(kJoinThreads), 0, s, a2, pairs));
        }
        if (dW) {
            rc = vk ? launch_product<true, true, kWeight>(m_u3, m_u3, m_scaled, m_dw, a3, pairs, s)
                    : launch_product<true, true, kWeight>(m_scaled, m_scaled, m_u3, m_dw, a3, pairs, s);
            if (rc) return rc;
        }
    }
    PPO_RETURN_IF_CUDA(launch_dependent(loss_kernel, dim3(1), dim3(kLossThreads), 0, s, r));
    return PPO_OK;
}
