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
// A row's reference is set before product 1, from the mean of 64 neighbouring logits, and serves columns whose largest y lies
// between 32 below and 96 above that mean: U and its sums stay inside fp32's (and bf16's) exponents, for logits of any size. 128
// columns whose largest lies elsewhere move their own reference by multiples of 128; where a row's references differ, the columns
// with a smaller one are multiplied by 2^(difference), which is exact, before product 2 (what is then under 2^-126, less than
// 2^-62 of the row's largest, becomes 0). (With references at multiples of 64,
// whatever the row's logits, many rows had two: 1999 x 50277 x 1032 with logits near -90 took 704 us, 638 so.)
//
// Roundings to 16 bits: U, a H (with more than 64 rows), and the results. Statistics, sums and nll are fp32, the loss fp64. What the rounding of U
// would do to the gradients is kept small in two ways. S in the gradient is the sum of the rounded U, so that D is the
// gradient of a softmax whose probabilities are off by half a step each and still add up to 1. U' at the label, about -S, is the
// largest element of its row by far: its own rounding is undone by a factor on a that makes a U' exact there, at the cost of
// that half step in the row's other elements. The row of D then adds up to c = a (exact - rounded) instead of 0, which would
// bring in what all columns of W have in common (logits far from 0 come from there); product 2 adds c times the mean of some
// columns of W to take that out again.
//
// Product kernel: persistent pairs of blocks (cta_group::2) on 256 x 256 tiles; per block one TMA producer warp (stages of
// 64 along the contraction, 128-byte swizzle), in the leader one issuer warp, eight epilogue warps in two groups that drain one
// 256-column accumulator while the next is formed. Operands are read as they lie in memory, K-major or MN-major, so that W may be
// stored [K, V] or [V, K].
//
// Bounds and times (calls one after the other): 27136 x 50304 x 4096 24.3 to 26.5 ms = 1260 to 1380 TFLOP/s, held by the board's
// power (about 1.4 GHz); three bare library products of these shapes take 24 ms there. At full clock L2 bounds the pairs (13.4 TB/s into the SMs).
// 1792 rows 1.52 ms (1460 TFLOP/s). 53 rows 259 us: W is streamed twice (products 1 and 2, 72 us each) and dW written once (78 us), 5.5 TB/s.
#include "ppo_tcgen05.cuh"

namespace ppo {
namespace xent {

using namespace tc;

constexpr int kBM = 128, kBlockK = 64, kBox = 64 * kBlockK * 2;
constexpr int kEpiWarps = 8, kThreads = (4 + kEpiWarps) * 32;
constexpr int kStageOut = 32 * 128;                        // a staging buffer: 32 rows x 64 bf16
constexpr int kChunk = 128;                                // columns with one reference
constexpr int kMaxSms = 160;
constexpr float kNoRef = -1.0e30f;
// 2^-64 and 2^64: the largest of a chunk's U lies between them, its smaller ones down to 2^-126 and their sums stay normal numbers
constexpr float kLeast = 5.421010862427522e-20f, kMost = 1.8446744073709552e19f;

// kPair: pairs of blocks share a tile of 256 x 256: each loads half of either operand and keeps half of the rows; one accumulator
// is drained while the next is formed.
// kWide: 256 x 512, both accumulators one tile's: a quarter less comes out of L2 per product (which bounds pairs: 64 KB in the
// 512 cycles of a block of the contraction are all that an SM's port takes), but draining them is not hidden. For long
// contractions.
// kSingle: blocks alone on tiles of 128 x 128, for up to 128 rows: half of a pair's tile would be idle rows, the tensor cores would
// take longer over them than memory over W, and there are too few wide tiles to share out evenly (197 of 256 columns at V =
// 50304, on 148 SMs: 101 us for product 1 of 53 rows, now 88). What bounds them is how much of W is on its way: more stages, and one
// staging buffer a warp (53 x 50304 x 4096 in all: 3 stages 302 us, 4 279, 5 266).
// kSmall: the same for products 1 and 2 of up to 64 rows: a stage holds 64 rows of A, so that there are eight. The matrix
// instruction reads 128: the other 64 rows are what lies behind them (B), and their results are nobody's.
// kTwice: pairs, for product 3 of up to 64 rows, with a H as the sum of two bf16 numbers: a stage holds both, and both are multiplied with
// the same U. With one block of contraction the products are hidden by the stores of dW (for 65 to 128 rows the whole call would take 3 to 5 %
// longer, beyond that a third), and what rounding a H once does to dW, as much as rounding dW itself, is gone: 53 x 50304 x 4096 dW 0.0024
// of its norm off with one, 0.0017 so, in the same 259 us; 53 x 50304 x 1064 109 and 113 us. (Blocks alone, which read half as much again
// out of L2: 265 and 112.)
enum Mode { kSingle, kPair, kWide, kSmall, kTwice };

template <int MODE>
struct Shape {
    static constexpr bool kIsPair = MODE == kPair || MODE == kWide || MODE == kTwice;
    static constexpr int kHalves = MODE == kWide ? 2 : 1;              // accumulators of a tile
    static constexpr int kM = kIsPair ? 2 * kBM : kBM, kAccN = kIsPair ? 256 : 128, kN = kHalves * kAccN;
    static constexpr int kRowsB = 128;                                 // a block's share of B, per accumulator
    static constexpr int kBytesA = (MODE == kSmall ? 64 : kBM) * kBlockK * 2, kBytesB = kRowsB * kBlockK * 2;
    static constexpr int kSecond = kBytesA + kHalves * kBytesB;        // where the second part of a H lies
    static constexpr int kStage = kSecond + (MODE == kTwice ? kBytesA : 0);
    static constexpr int kStages = MODE == kWide || MODE == kTwice ? 4 : MODE == kPair ? 5 : MODE == kSingle ? 6 : 8;
    static constexpr int kBuffers = MODE == kPair ? 2 : 1;             // staging, per epilogue warp
    static constexpr int kSmem = kStages * kStage + kBuffers * kEpiWarps * kStageOut + 1024;
    static constexpr int kTileFloats = kM * kN;
    static_assert(kSmem <= 232448 - 1024, "shared memory of a block");
};

enum Product { kLogits = 1, kHidden = 2, kWeight = 3 };

struct Args {
    // rows of this piece: min(rows_max, max(0, *n_real - row0)), known on the device
    const int *n_real;
    int M, row0, rows_max;
    int dim_m, dim_n, dim_k;                               // result [dim_m, dim_n], contraction dim_k; the rows' one is an upper bound
    int gm, gn;
    int *status;
    // kLogits
    int in_place;                                          // H may be read where it lies
    const int32_t *order;                                  // order[i]: the original row of real row i
    const int4 *info;                                      // [M] of real row i: label; as bits: reference, log2(e) / tau, `cut`
    float *picked;                                         // [rows] accumulator at the label
    float4 *part;                                          // [rows][chunks] reference, sum, sum of the rounded values
    int chunks, store;
    // results
    __nv_bfloat16 *out;
    int64_t ldo;
    int bulk_cols;                                         // bulk stores take boxes that end at or before this column
    // kTwice
    int vk, second;                                        // a H is B (else A); first row of its second part
    // kHidden
    const float2 *row_scale;                               // [rows] a, c
    const float *w_mean;                                   // [K, in whole tiles]
    const int2 *slices;                                    // of the tiles that are left over, and their length
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

template <int STAGES>
struct Smem {
    unsigned long long full[STAGES], empty[STAGES], tmem_full[2], tmem_empty[2];
    uint32_t tmem_base;
};

// The workers (pairs, or blocks) take tiles 0 .. n_whole in turn, whole, and then the slices along the contraction of the other
// tiles, which are too few for all workers: first slices of all of them, second slices, ... so that workers that run at the
// same time read the same blocks of their operands, through L2. (Cut end to end into equal shares, with each worker at a
// place of its own, 38 tiles over for 74 pairs came at 1100 cycles a block instead of 600, from memory.) A slice's sums go
// to scratch, and join_kernel adds them up in order.
struct Plan {
    int m_tiles, n_tiles, n_whole, n_rest, slices, length, kbs;     // length: of a slice, in blocks of the contraction
};

template <int MODE, int PRODUCT>
__device__ __forceinline__ Plan plan_of(const Args &a, int rows, int workers)
{
    constexpr int kM = Shape<MODE>::kM;
    Plan p;
    p.m_tiles = ((PRODUCT == kWeight ? a.dim_m : rows) + kM - 1) / kM;
    p.n_tiles = (a.dim_n + Shape<MODE>::kN - 1) / Shape<MODE>::kN;
    p.kbs = ((PRODUCT == kWeight ? rows : a.dim_k) + kBlockK - 1) / kBlockK;
    p.n_whole = p.m_tiles * p.n_tiles;
    p.n_rest = 0;
    p.slices = 1;
    p.length = p.kbs;
    if (PRODUCT == kWeight && rows == 0 && a.row0 > 0) p.n_whole = 0;      // nothing to add
    if (PRODUCT == kHidden && a.slices->x > 1) {
        p.n_rest = p.n_whole % workers;
        p.slices = a.slices->x;
        p.length = a.slices->y;
        p.n_whole -= p.n_rest;
    }
    return p;
}

struct Work {
    int u, kb0, kb1;      // tile, blocks of the contraction
    int part;             // -1: whole; else the slice's place in scratch
    int next_unit;
    __device__ __forceinline__ void init(int worker) { next_unit = worker; }
    __device__ __forceinline__ bool next(const Plan &p, int workers)
    {
        u = next_unit;
        part = u - p.n_whole;
        next_unit += workers;
        kb0 = 0;
        kb1 = p.kbs;
        if (part < 0) {
            part = -1;
            return true;
        }
        if (part >= p.n_rest * p.slices) return false;
        const int slice = part / p.n_rest;
        u = p.n_whole + part - slice * p.n_rest;
        kb0 = slice * p.length;
        kb1 = min(p.kbs, kb0 + p.length);
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

// eight neighbouring columns of this lane's row, the c8-th of the buffer's 64
__device__ __forceinline__ void stage8(unsigned char *stage, int c8, const uint32_t *w)
{
    const int lane = threadIdx.x & 31;
    *reinterpret_cast<uint4 *>(stage + lane * 128 + ((c8 ^ (lane & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
}

// 64 columns
__device__ __forceinline__ void stage64(unsigned char *stage, const float *v)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack2(v[j * 8 + e * 2], v[j * 8 + e * 2 + 1]);
        stage8(stage, j, w);
    }
}

template <int MODE, bool A_MN, bool B_MN, int PRODUCT>
__global__ void __launch_bounds__(kThreads, 1)
product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_a_all,
               const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_out, const Args a)
{
    using S = Shape<MODE>;
    static_assert(MODE != kSmall || !A_MN, "rows of A are what there are few of");
    static_assert(MODE != kTwice || (A_MN && B_MN && S::kBytesA == S::kBytesB), "either operand may be the one in two parts");
    constexpr bool PAIR = S::kIsPair;
    constexpr int kStages = S::kStages, kHalves = S::kHalves;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ Smem<kStages> sm;
    unsigned char *ring = smem_raw + ((1024u - (saddr(smem_raw) & 1023u)) & 1023u);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            barrier_init(&sm.full[s], 1);
            barrier_init(&sm.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            barrier_init(&sm.tmem_full[b], 1);
            barrier_init(&sm.tmem_empty[b], (PAIR ? 2 : 1) * kEpiWarps / 2);     // a group of each block
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        if (PAIR) tmem_alloc_all_pair(&sm.tmem_base);
        else tmem_alloc_all(&sm.tmem_base);
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (PAIR) cluster_barrier();                                // the other block's barriers are ready too
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = sm.tmem_base;
    // (in this order: what the launches before this one wrote is there when row_kernel starts)
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int rank = PAIR ? (int)cluster_rank() : 0;
    const int worker = PAIR ? blockIdx.x / 2 : blockIdx.x, workers = PAIR ? gridDim.x / 2 : gridDim.x;
    const int rows = rows_of(a);
    const Plan plan = plan_of<MODE, PRODUCT>(a, rows, workers);
    Work work;
    work.init(worker);

    if (warp == 0) {
        if (lane == 0) {
            // (where all rows are real they need not have been packed)
            const CUtensorMap *ma = PRODUCT == kLogits && a.in_place && *a.n_real == a.M ? &map_a_all : &map_a;
            const int row0 = PRODUCT == kLogits ? a.row0 : 0;
            const uint32_t full0 = PAIR ? leader_addr(&sm.full[0]) : 0;
            bool alive = true;
            uint32_t it = 0, s = 0, parity = 1;                 // (waiting for the phase before the first returns at once)
            while (alive && work.next(plan, workers)) {
                const int2 t = tile_of(work.u, plan.m_tiles, plan.n_tiles, a.gm, a.gn);
                const int m0 = t.x * S::kM + rank * kBM, n0 = t.y * S::kN + rank * S::kRowsB;
                for (int kb = work.kb0; kb < work.kb1; ++kb, ++it) {
                    wait_alive(alive, &sm.empty[s], parity, a.status);
                    if (!alive) break;
                    unsigned char *stage = ring + (size_t)s * S::kStage;
                    // (bytes of the other block may be counted before they are announced: the phase cannot end
                    // without the leader's arrival)
                    if (rank == 0) barrier_expect_tx(&sm.full[s], (PAIR ? 2u : 1u) * S::kStage);
                    const uint32_t bar = full0 + s * 8;
                    const auto load = [&](unsigned char *dst, const CUtensorMap *map, int x, int y) {
                        if (PAIR) tma_load_2d_pair(dst, map, x, y, bar);
                        else tma_load_2d(dst, map, x, y, &sm.full[s]);
                    };
                    if (A_MN) {                                 // stored [k, m]: boxes of 64 (m) x 64 (k)
                        load(stage, ma, m0, kb * kBlockK);
                        load(stage + kBox, ma, m0 + 64, kb * kBlockK);
                    } else {                                    // stored [m, k]: one box of 64 (k) x 128 (m)
                        load(stage, ma, kb * kBlockK, row0 + m0);
                    }
#pragma unroll
                    for (int i = 0; i < kHalves; ++i) {
                        unsigned char *to = stage + S::kBytesA + i * S::kBytesB;
                        if (B_MN) {
                            load(to, &map_b, n0 + i * S::kAccN, kb * kBlockK);
                            load(to + kBox, &map_b, n0 + i * S::kAccN + 64, kb * kBlockK);
                        } else {
                            load(to, &map_b, kb * kBlockK, n0 + i * S::kAccN);
                        }
                    }
                    if (MODE == kTwice) {
                        const CUtensorMap *map = a.vk ? &map_b : ma;
                        const int x = a.vk ? n0 : m0, y = a.second + kb * kBlockK;
                        load(stage + S::kSecond, map, x, y);
                        load(stage + S::kSecond + kBox, map, x + 64, y);
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
            constexpr uint32_t idesc = instr_desc(A_MN, B_MN, S::kM, S::kAccN);
            // K-major: 8-row groups 1024 bytes apart; MN-major: 64-wide boxes, 8 contraction rows 1024 bytes apart. (A stage is added
            // to descriptors made once: the thread's own instructions, which take turns with those of two epilogue warps,
            // otherwise take longer than the products.)
            const uint64_t a_desc = smem_desc(saddr(ring), A_MN ? kBox : 16, 1024);
            const uint64_t b_desc = smem_desc(saddr(ring) + S::kBytesA, B_MN ? kBox : 16, 1024);
            const auto announce = [](unsigned long long *bar) {
                if (PAIR) commit_pair(bar);
                else commit(bar);
            };
            bool alive = true;
            uint32_t s = 0, s_parity = 0, tiles = 0;
            // one block of the contraction into accumulator `acc`, from stage `from`
            const uint32_t a_second = a.vk ? 0 : S::kSecond >> 4, b_second = a.vk ? (S::kSecond - S::kBytesA) >> 4 : 0;
            const auto multiply = [&](uint32_t acc, uint32_t from, int half, uint32_t accumulate) {
                const uint64_t ad = a_desc + from * (S::kStage >> 4), bd = b_desc + (from * S::kStage + half * S::kBytesB >> 4);
#pragma unroll
                for (int kk = 0; kk < kBlockK / 16; ++kk) {
                    // 16 contraction elements further: 32 bytes K-major, 16 rows of 128 MN-major
                    const uint64_t ak = ad + kk * (A_MN ? 2048 >> 4 : 32 >> 4), bk = bd + kk * (B_MN ? 2048 >> 4 : 32 >> 4);
                    if (PAIR) mma_pair(tmem_base + acc * S::kAccN, ak, bk, idesc, kk ? 1u : accumulate);
                    else mma(tmem_base + acc * S::kAccN, ak, bk, idesc, kk ? 1u : accumulate);
                    if (MODE == kTwice) mma_pair(tmem_base + acc * S::kAccN, ak + a_second, bk + b_second, idesc, 1u);
                }
            };
            const auto step = [&] { if (++s == kStages) { s = 0; s_parity ^= 1; } };
            while (alive && work.next(plan, workers)) {
                int kb = work.kb0;
                if (kb == work.kb1) continue;                   // an empty contraction: the epilogue knows
                const uint32_t buf = kHalves == 2 ? 0 : tiles & 1, parity = (kHalves == 2 ? tiles & 1 : tiles >> 1 & 1) ^ 1;
                wait_alive(alive, &sm.tmem_empty[buf], parity, a.status);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (kHalves == 2) {
                    // the first accumulator goes ahead, as far as the stages reach, while the second one is drained
                    const uint32_t s0 = s, p0 = s_parity;
                    const int lead = min(work.kb1 - kb, kStages);
                    for (int i = 0; i < lead && alive; ++i) {
                        wait_alive(alive, &sm.full[s], s_parity, a.status);
                        if (!alive) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        multiply(0, s, 0, i ? 1u : 0u);
                        step();
                    }
                    wait_alive(alive, &sm.tmem_empty[1], parity, a.status);
                    if (!alive) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    s = s0;
                    s_parity = p0;
                    if (lead == work.kb1 - kb && PPO_TEST_WITHHOLD_XENT != 1) announce(&sm.tmem_full[0]);
                    for (int i = 0; i < lead; ++i) {
                        multiply(1, s, 1, i ? 1u : 0u);
                        announce(&sm.empty[s]);
                        step();
                    }
                    kb += lead;
                }
                for (; kb < work.kb1; ++kb) {
                    wait_alive(alive, &sm.full[s], s_parity, a.status);
                    if (!alive) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    multiply(buf, s, 0, kb > work.kb0 ? 1u : 0u);
                    if (kHalves == 2) {
                        if (kb == work.kb1 - 1 && PPO_TEST_WITHHOLD_XENT != 1) announce(&sm.tmem_full[0]);
                        multiply(1, s, 1, 1u);
                    }
                    announce(&sm.empty[s]);
                    step();
                }
                if (alive && PPO_TEST_WITHHOLD_XENT != 1) {
                    announce(&sm.tmem_full[kHalves == 2 ? 1 : buf]);
                    ++tiles;
                }
            }
            // every product has ended before tensor memory is freed, and the other block's last arrivals before this block ends
            if (kHalves == 2) {
                for (int i = 0; i < 2 && tiles > 0; ++i) wait(&sm.tmem_full[i], (tiles - 1) & 1, a.status);
                for (int i = 0; i < 2 && tiles > 0; ++i) wait_alive(alive, &sm.tmem_empty[i], (tiles - 1) & 1, a.status);
            } else {
                for (uint32_t i = tiles > 2 ? tiles - 2 : 0; i < tiles; ++i) wait(&sm.tmem_full[i & 1], (i >> 1) & 1, a.status);
                for (uint32_t i = tiles > 2 ? tiles - 2 : 0; i < tiles; ++i)
                    wait_alive(alive, &sm.tmem_empty[i & 1], (i >> 1) & 1, a.status);
            }
        }
        __syncwarp();
    } else if (warp >= 4) {
        // lanes 32 q .. of every second accumulator: two groups of warps take turns, so that what a tile costs beside its columns
        // (waits, loads, copies) falls into the other group's time
        const int q = warp & 3, group = (warp - 4) >> 2;
        unsigned char *const stage = ring + (size_t)kStages * S::kStage + (warp - 4) * S::kBuffers * kStageOut;
        const uint32_t tmem_empty = PAIR ? leader_addr(&sm.tmem_empty[0]) : saddr(&sm.tmem_empty[0]);
        const float nan = __int_as_float(0x7fffffff);
        const bool first = a.row0 == 0, last = a.row0 + a.rows_max >= *a.n_real;
        bool alive = true;
        uint32_t tiles = 0;
        // (a wide tile's accumulators one after the other)
        for (int part_of = kHalves; part_of < kHalves || work.next(plan, workers); ++tiles) {
            const int half_tile = kHalves == 2 ? tiles & 1 : 0;
            part_of = half_tile + 1;
            if ((int)(tiles & 1) != group) continue;
            const int2 t = tile_of(work.u, plan.m_tiles, plan.n_tiles, a.gm, a.gn);
            const int m_warp = t.x * S::kM + rank * kBM + q * 32, n_tile = t.y * S::kN + half_tile * S::kAccN;
            const int row = m_warp + lane;
            const bool empty = work.kb0 == work.kb1;
            const uint32_t buf = tiles & 1;
            bool ok = false;
            int label_tile = -1, out_row = -1;
            float ref_row = 0.f, c = 0.f;
            float2 scale = make_float2(0.f, 0.f);
            if (PRODUCT == kLogits) {
                ok = row < rows;
                if (ok) {
                    const int4 info = a.info[a.row0 + row];
                    label_tile = (int)((unsigned)info.x - (unsigned)n_tile);
                    ref_row = __int_as_float(info.y);
                    c = __int_as_float(info.z);
                }
            } else if (PRODUCT == kHidden) {
                ok = row < rows;
                if (ok && work.part < 0) {
                    out_row = a.order[a.row0 + row];
                    scale = a.row_scale[row];
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
#pragma unroll 1
            for (int h = 0; h < S::kAccN / 128; ++h) {              // 128 columns
                const int n = n_tile + h * 128, label = label_tile - h * 128;
                const bool last_read = h == S::kAccN / 128 - 1;
                const uint32_t taddr = tmem_base + buf * S::kAccN + h * 128 + ((uint32_t)(q * 32) << 16);
                float ref = ref_row;
                // 64 columns of this lane's row
                const auto read = [&](int half, float (&v)[64]) {
                    if (empty || !alive) {
#pragma unroll
                        for (int j = 0; j < 64; ++j) v[j] = alive ? 0.f : nan;
                        return;
                    }
                    uint32_t r0[32], r1[32];
                    __syncwarp();
                    tmem_ld32(taddr + half * 64, r0);
                    tmem_ld32(taddr + half * 64 + 32, r1);
                    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        v[j] = __uint_as_float(r0[j]);
                        v[j + 32] = __uint_as_float(r1[j]);
                    }
                };
                const auto release = [&] {                          // nothing of the accumulator is needed any more
                    if (empty) return;
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    const bool arrive = lane == 0 && alive && PPO_TEST_WITHHOLD_XENT != 2;
                    if (PAIR) barrier_arrive_cluster_if(tmem_empty + buf * 8, arrive);
                    else if (arrive) barrier_arrive(&sm.tmem_empty[buf]);
                };
                // the staging buffers, whose last copies have read them
                const auto reuse = [&] {
                    if (lane == 0) tma_store_wait_read();
                    __syncwarp();
                };
                // 64-column parts from .. to of these 128, from their buffers, by bulk copies as far as they may go
                const auto send = [&](int from, int to, int bulk_cols, bool rows_here) {
                    fence_async_proxy();
                    __syncwarp();
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int col = n + half * 64;
                        if (half < from || half >= to || col >= a.dim_n) continue;
                        const unsigned char *buffer = stage + (S::kBuffers == 2 ? half : 0) * kStageOut;
                        if (col + 64 <= bulk_cols) {
                            if (lane == 0 && rows_here) tma_store_2d(&map_out, col, m_warp, buffer);
                        } else {
                            store_rows(buffer, a.out, a.ldo, out_row, col, a.dim_n);
                        }
                    }
                    __syncwarp();
                };

                if (PRODUCT == kLogits) {
                    // U with the row's reference. Where a lane's largest value has left the window, once more with another one:
                    // with two staging buffers that is looked at when all 128 are there, with one for each 64 before they leave.
                    float s = 0.f, rounded = 0.f;
                    const bool plain = __all_sync(0xffffffffu, ok) && n + 128 <= a.dim_n;
#pragma unroll 1
                    for (int turn = 0; turn < 2; ++turn) {
                        float top = 0.f;
                        bool again = false;
                        s = rounded = 0.f;
#pragma unroll 1
                        for (int half = 0; half < 2; ++half) {
                            if (a.store && (S::kBuffers == 1 || half == 0)) reuse();
                            unsigned char *buffer = stage + (S::kBuffers == 2 ? half : 0) * kStageOut;
                            float v[64];
                            read(half, v);
                            if ((unsigned)(label - half * 64) < 64u) {
#pragma unroll
                                for (int j = 0; j < 64; ++j)
                                    if (label - half * 64 == j) a.picked[row] = v[j];
                            }
                            const int left = plain ? 64 : ok ? a.dim_n - n - half * 64 : 0;
                            float s1 = 0.f, r1 = 0.f;
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                uint32_t w[4];
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const int i = j * 8 + e * 2;
                                    float x = ex2(fmaf(v[i], c, -ref)), y = ex2(fmaf(v[i + 1], c, -ref));
                                    if (!plain) {
                                        x = i < left ? x : 0.f;
                                        y = i + 1 < left ? y : 0.f;
                                    }
                                    top = fmaxf(top, fmaxf(x, y));
                                    s += x;
                                    s1 += y;
                                    w[e] = pack2(x, y);
                                    rounded += low(w[e]);
                                    r1 += high(w[e]);
                                }
                                if (a.store) stage8(buffer, j, w);
                            }
                            s += s1;
                            rounded += r1;
                            // (a lane without a column has 0 everywhere)
                            if (turn == 0 && (S::kBuffers == 1 || half == 1)) {
                                const bool out = ok && n + (S::kBuffers == 1 ? half * 64 : 0) < a.dim_n && !(top >= kLeast && top <= kMost);
                                again = __any_sync(0xffffffffu, out);
                                if (again) break;
                            }
                            if (a.store && S::kBuffers == 1) send(half, half + 1, 0x7fffffff, true);
                        }
                        if (!again) break;
                        // (what has left has arrived before it is written again)
                        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
                        __syncwarp();
                        float m = kNoRef;
#pragma unroll 1
                        for (int half = 0; half < 2; ++half) {
                            float v[64];
                            read(half, v);
                            const int left = a.dim_n - n - half * 64;
#pragma unroll
                            for (int j = 0; j < 64; ++j) m = j < left ? fmaxf(m, v[j]) : m;
                        }
                        // (unchanged where the largest one is in the window)
                        if (ok) ref += 128.f * rintf((fmaxf(m * c, -1e9f) - ref) * (1.f / 128.f));
                    }
                    if (last_read) release();
                    if (a.store && S::kBuffers == 2) send(0, 2, 0x7fffffff, true);
                    if (ok && n < a.dim_n) a.part[(size_t)row * a.chunks + n / kChunk] = make_float4(ref, s, rounded, 0.f);
                } else if (PRODUCT == kHidden) {
                    // (four columns of a tile's rows follow one another in scratch: a warp writes 512 bytes at a time)
                    float4 *part = reinterpret_cast<float4 *>(a.scratch + (size_t)max(work.part, 0) * S::kTileFloats) +
                                   (half_tile * 64 + h * 32) * S::kM + rank * kBM + q * 32 + lane;
#pragma unroll 1
                    for (int half = 0; half < 2; ++half) {
                        float v[64];
                        read(half, v);
                        if (half == 1 && last_read) release();
                        if (work.part >= 0) {
                            if (!ok) continue;
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                part[(half * 16 + j) * S::kM] = make_float4(v[j * 4], v[j * 4 + 1], v[j * 4 + 2], v[j * 4 + 3]);
                            continue;
                        }
                        const float4 *mean = reinterpret_cast<const float4 *>(a.w_mean + n + half * 64);
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const float4 w = __ldg(mean + j);
                            v[j * 4] = fmaf(v[j * 4], scale.x, scale.y * w.x);
                            v[j * 4 + 1] = fmaf(v[j * 4 + 1], scale.x, scale.y * w.y);
                            v[j * 4 + 2] = fmaf(v[j * 4 + 2], scale.x, scale.y * w.z);
                            v[j * 4 + 3] = fmaf(v[j * 4 + 3], scale.x, scale.y * w.w);
                        }
                        stage64(stage + (S::kBuffers == 2 ? half : 0) * kStageOut, v);
                        send(half, half + 1, 0, true);
                    }
                } else {
                    float4 *sum = reinterpret_cast<float4 *>(a.scratch + ((size_t)t.x * plan.n_tiles + t.y) * S::kTileFloats) +
                                  (half_tile * 64 + h * 32) * S::kM + rank * kBM + q * 32 + lane;
                    if (last && S::kBuffers == 2) reuse();
#pragma unroll 1
                    for (int half = 0; half < 2; ++half) {
                        float v[64];
                        read(half, v);
                        if (half == 1 && last_read) release();
                        if (!first) {
                            float4 old[16];
#pragma unroll
                            for (int j = 0; j < 16; ++j) old[j] = sum[(half * 16 + j) * S::kM];
#pragma unroll
                            for (int j = 0; j < 16; ++j) {
                                v[j * 4] += old[j].x; v[j * 4 + 1] += old[j].y; v[j * 4 + 2] += old[j].z; v[j * 4 + 3] += old[j].w;
                            }
                        }
                        if (last) {
                            if (S::kBuffers == 1) reuse();
                            stage64(stage + (S::kBuffers == 2 ? half : 0) * kStageOut, v);
                            if (S::kBuffers == 1 || half == 1) send(S::kBuffers == 1 ? half : 0, half + 1, a.bulk_cols, m_warp < a.dim_m);
                        } else {
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                sum[(half * 16 + j) * S::kM] = make_float4(v[j * 4], v[j * 4 + 1], v[j * 4 + 2], v[j * 4 + 3]);
                        }
                    }
                }
            }
        }
        if (lane == 0) tma_store_wait_read();                   // shared memory outlives the copies out of it
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (PAIR) cluster_barrier();                                // neither block ends while the other may reach into it
    if (warp == 0) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (PAIR) tmem_free_all_pair(tmem_base);
        else tmem_free_all(tmem_base);
    }
}

// The tiles of dH that were cut along the vocabulary: a block adds up 32 rows x 64 columns of their slices, in order, and turns
// them in shared memory so that rows leave in runs.
constexpr int kJoinThreads = 256;
template <int MODE> constexpr int join_blocks() { return (Shape<MODE>::kM / 32) * (Shape<MODE>::kN / 64); }
template <int MODE>
__device__ __forceinline__ void join_tiles(const Args &a, int workers, int block)
{
    constexpr int kM = Shape<MODE>::kM, kTileFloats = Shape<MODE>::kTileFloats, kBlocks = (kM / 32) * (Shape<MODE>::kN / 64);
    __shared__ float4 turn[32][17];
    const int rows = rows_of(a);
    const Plan p = plan_of<MODE, kHidden>(a, rows, workers);
    const int rest = block / kBlocks, part_of = block % kBlocks;
    if (rest >= p.n_rest) return;
    const int row0 = (part_of % (kM / 32)) * 32, j0 = part_of / (kM / 32) * 16;
    const int2 t = tile_of(p.n_whole + rest, p.m_tiles, p.n_tiles, a.gm, a.gn);
    const int m0 = t.x * kM + row0, n0 = t.y * Shape<MODE>::kN + j0 * 4;
    if (m0 >= rows || n0 >= a.dim_n) return;
    const int lane = threadIdx.x & 31, jj = threadIdx.x >> 5;
    float4 v[2];
    v[0] = v[1] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int i = 0; i < p.slices; ++i) {
        const float4 *from = reinterpret_cast<const float4 *>(a.scratch + (size_t)(i * p.n_rest + rest) * kTileFloats) + row0 + lane;
        const float4 x = from[(j0 + jj) * kM], y = from[(j0 + jj + 8) * kM];
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
        const float4 w = *reinterpret_cast<const float4 *>(a.w_mean + n);
        const float y[4] = {fmaf(x.x, s.x, s.y * w.x), fmaf(x.y, s.x, s.y * w.y), fmaf(x.z, s.x, s.y * w.z), fmaf(x.w, s.x, s.y * w.w)};
        __nv_bfloat16 *to = a.out + (int64_t)a.order[a.row0 + m0 + r] * a.ldo + n;
        if (n + 4 <= a.dim_n && reinterpret_cast<uintptr_t>(to) % 8 == 0) {
            *reinterpret_cast<uint2 *>(to) = make_uint2(pack2(y[0], y[1]), pack2(y[2], y[3]));
        } else {
            for (int e = 0; e < 4 && n + e < a.dim_n; ++e) to[e] = __float2bfloat16_rn(y[e]);
        }
    }
}

template <int MODE>
__global__ void __launch_bounds__(kJoinThreads)
join_kernel(const Args a, int workers)
{
    grid_dependents_may_launch();
    grid_dependency_wait();
    join_tiles<MODE>(a, workers, blockIdx.x);
}

// ---------------------------------------------------------------- rows
struct RowArgs {
    const __nv_bfloat16 *H;
    int64_t ldh, lddh;
    int M, K, V, Kp;                                            // Kp: row pitch of the packed and the scaled rows
    const int32_t *labels;
    const uint8_t *mask;
    int32_t ignore_id;
    double c;                                                   // log2(e) / tau
    float inv_tau, scale;
    const float *denom;
    int32_t *order;                                             // [M] real rows, ascending; then the others
    int *n_real;
    const __nv_bfloat16 *W;
    int64_t ldw;
    int vk;
    float *w_mean, *w_one;                                      // [K] mean of kSample columns of W, and the first of them
    int4 *info;                                                 // [M] of real row i: label, reference, its c, what its logits have lost, all alike
    int in_place;                                               // product 1 reads H where it lies when all rows are real
    __nv_bfloat16 *packed;                                      // [M, Kp] real rows (unless they can be read in place)
    __nv_bfloat16 *scaled;                                      // [rows_max, Kp] a H; null: no gradients
    int64_t second;                                             // 0, or elements from there to what its rounding leaves, rounded
    __nv_bfloat16 *u;                                           // [rows_max, Vp]
    int64_t Vp;
    float *picked;
    float2 *row_scale;
    float4 *part;
    int chunks, row0, rows_max;
    int tile_m, n_tiles, workers, kbs;                          // product 2: tile rows, tiles along K, workers, blocks along V
    int2 *slices;
    float *loss, *nll, *lse;
    __nv_bfloat16 *dH;
    int *status;
};

// The mean of kSample neighbouring columns of W, from the middle of the vocabulary, and the first one, for some hidden elements: a thread loads
// eight neighbours in memory, eight (stored [K, V]) or 64 (stored [V, K]) threads share an element. (One element after the
// other, 64 loads each: 36 us at K = 4096, most of it misses of the address translation.)
constexpr int kOrderThreads = 1024, kOrderPer = 8, kSample = 64, kMeanPer = kOrderThreads / 8;
__device__ __forceinline__ void mean_columns(const RowArgs &a, int k0, float (*part)[kMeanPer])
{
    const int v0 = min(a.V / 2, max(0, a.V - kSample)) & ~7, n = min(kSample, a.V - v0);
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (a.vk) {
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
            if (j == 0)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (k + e < a.K) a.w_one[k + e] = x[e];
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
        if (v == v0) a.w_one[k] = __bfloat162float(w[0]);
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
// What the tensor cores cut off. After every 16 elements of the contraction they keep the sum to a quarter of its last place and
// then to its last place, 3/8 of it on average (measured): 3 * 2^-26 of the sum's power of two. A logit that grows evenly passes through
// sums whose powers of two average 0.36 of it, and loses 0.36 * 3 * 2^-26 / 16 = 1.0e-9 of itself for each element (measured: 0.9e-9 to
// 1.1e-9 for K = 1024 to 131072 and logits up to 20; 1.4e-9 where all products have one sign). Nothing is lost where nothing can be: 16 elements
// whose products (with a column of W that stands for all) are multiples of the last place of the sum of the absolute products so far
// are not counted; such sums are exact whatever their order. Elements that are 0, in H or in W, are the plainest case.
constexpr float kCutStep = 4.4703484e-8f;
constexpr double kCutEven = 1.0e-9;
constexpr unsigned kCutMost = 1u << 17;                        // elements: as far as it has been measured
// real rows: label, reference and what they lose, and a packed copy where they are not read in place; the rows left out get their zeros
__global__ void __launch_bounds__(kRowThreads)
pack_kernel(const RowArgs a)
{
    constexpr int kWarps = kRowThreads / 32;
    __shared__ float red[2][kWarps];
    __shared__ unsigned red_n[kWarps];
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
    const bool pack = n < a.M || !a.in_place;
    // Product with the mean column, and beside it what is cut off of the sums that all columns have in common.
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float before = 0.f, cut = 0.f, all = 0.f;                   // ahead of these 2048 elements: the sum, the absolute one; powers of two cut from
    unsigned groups = 0;                                        // of 16 elements that cut
    for (int k = threadIdx.x * 8, k0 = 0; k0 < a.K; k += kRowThreads * 8, k0 += kRowThreads * 8) {
        float s = 0.f, size = 0.f, one[8];                      // `one`: products with a single column
#pragma unroll
        for (int e = 0; e < 8; ++e) one[e] = 0.f;
        if (k + 8 <= a.K) {
            const uint4 v = *reinterpret_cast<const uint4 *>(from + k);
            if (pack) *reinterpret_cast<uint4 *>(to + k) = v;
            const float4 p = *reinterpret_cast<const float4 *>(a.w_mean + k), q = *reinterpret_cast<const float4 *>(a.w_mean + k + 4);
            s = fmaf(low(v.x), p.x, s); s = fmaf(high(v.x), p.y, s); s = fmaf(low(v.y), p.z, s); s = fmaf(high(v.y), p.w, s);
            s = fmaf(low(v.z), q.x, s); s = fmaf(high(v.z), q.y, s); s = fmaf(low(v.w), q.z, s); s = fmaf(high(v.w), q.w, s);
            const float4 x = *reinterpret_cast<const float4 *>(a.w_one + k), y = *reinterpret_cast<const float4 *>(a.w_one + k + 4);
            one[0] = low(v.x) * x.x; one[1] = high(v.x) * x.y; one[2] = low(v.y) * x.z; one[3] = high(v.y) * x.w;
            one[4] = low(v.z) * y.x; one[5] = high(v.z) * y.y; one[6] = low(v.w) * y.z; one[7] = high(v.w) * y.w;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (k + e >= a.K) break;
                if (pack) to[k + e] = from[k + e];
                const float h = __bfloat162float(from[k + e]);
                s = fmaf(h, a.w_mean[k + e], s);
                one[e] = h * a.w_one[k + e];
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) size += fabsf(one[e]);
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const float o = __shfl_up_sync(0xffffffffu, s, off), p = __shfl_up_sync(0xffffffffu, size, off);
            if (lane >= off) {
                s += o;
                size += p;
            }
        }
        if (lane == 31) {
            red[0][warp] = s;
            red[1][warp] = size;
        }
        __syncthreads();
        float ahead = before;
        size += all;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) {
                ahead += red[0][w];
                size += red[1][w];
            }
            before += red[0][w];
            all += red[1][w];
        }
        // a number is a multiple of the last place of a power of two where 1.5 times that, added and taken off, leaves it alone
        const float power = 1.5f * __int_as_float(__float_as_int(size) & 0x7f800000);
        bool cuts = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) cuts |= __fsub_rn(__fadd_rn(one[e], power), power) != one[e];
        const unsigned group = __ballot_sync(0xffffffffu, cuts) >> (lane & 30) & 3u;
        if (group && k < a.K && (lane & 1 || k + 8 >= a.K)) {
            cut += __int_as_float(__float_as_int(ahead + s) & 0xff800000);
            ++groups;
        }
        __syncthreads();
    }
    cut = warp_sum_f(cut);
    groups = __reduce_add_sync(0xffffffffu, groups);
    if (lane == 0) {
        red[0][warp] = cut;
        red_n[warp] = groups;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        float s = before;
        cut = 0.f;
        groups = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            cut += red[0][w];
            groups += red_n[w];
        }
        // by a factor, what logits lose that grow evenly; to lse, what the common part has lost beyond that
        const double even = kCutEven * 16.0 * (double)min(groups, kCutMost / 16);
        const float c = (float)(a.c * (1.0 + even));
        cut = (cut * kCutStep - (float)even * s) * a.inv_tau;
        // the middle of the window; whole numbers, so that y - reference loses nothing that y does not
        s = rintf(s * c) + 32.f;
        a.info[i] = make_int4(a.labels[row], __float_as_int(fabsf(s) < 1e9f ? s : 0.f), __float_as_int(c),
                              __float_as_int(fabsf(cut) < 1.f ? cut : 0.f));
    }
}

// How the tiles of product 2 that are too few for all workers are sliced: rounds x length, and for the joining 20 blocks' time
// and that of one block for six slices, is least; scratch holds two tiles a worker. By one block, a thread for each number.
__device__ __forceinline__ void choose_slices(const RowArgs &a, int rows)
{
    __shared__ unsigned best[kRowThreads / 32];
    const int rest = (rows + a.tile_m - 1) / a.tile_m * a.n_tiles % a.workers;
    unsigned mine = (unsigned)min(a.kbs, 1 << 20) << 10 | 1u;           // whole
    for (int s = threadIdx.x + 2; rest > 0 && rest * s <= 2 * a.workers && s <= a.kbs; s += kRowThreads) {
        const int length = (a.kbs + s - 1) / s, n = (a.kbs + length - 1) / length;       // (none empty)
        const int cost = (rest * n + a.workers - 1) / a.workers * length + 20 + rest * n / 6;
        mine = min(mine, (unsigned)min(cost, 1 << 20) << 10 | (unsigned)n);
    }
    mine = __reduce_min_sync(0xffffffffu, mine);
    if ((threadIdx.x & 31) == 0) best[threadIdx.x >> 5] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kRowThreads / 32; ++w) mine = min(mine, best[w]);
        const int n = (int)(mine & 1023u), length = (a.kbs + n - 1) / n;
        *a.slices = make_int2(n, length);
    }
}

// what rounding x leaves; nothing where that is no number
__device__ __forceinline__ float left_over(float x, float rounded)
{
    const float d = x - rounded;
    return fabsf(d) < __int_as_float(0x7f800000) ? d : 0.f;
}

// A row's statistics out of its chunks', its loss and the factors of its gradient; U at the label; a H
__global__ void __launch_bounds__(kRowThreads)
row_kernel(const RowArgs a)
{
    __shared__ float red[3][kRowThreads / 32];
    // What this kernel needs and product 1 does not write is loaded while that still runs: a chain of three loads from memory.
    const int n_real = __ldcg(a.n_real), rows = max(0, min(a.rows_max, n_real - a.row0)), r = (int)blockIdx.x - 1;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int row = 0;
    int4 info = make_int4(-1, 0, 0, 0);
    uint4 ahead[2] = {};                                        // of the row of H: this thread's first two pieces of eight
    const __nv_bfloat16 *h = a.H;
    if (r >= 0 && r < rows) {
        row = __ldcg(a.order + a.row0 + r);
        info = __ldcg(a.info + a.row0 + r);
        h += (int64_t)row * a.ldh;
        if (a.scaled) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int k = (j * kRowThreads + threadIdx.x) * 8;
                if (k + 8 <= a.K) ahead[j] = __ldcg(reinterpret_cast<const uint4 *>(h + k));
            }
        }
    }
    grid_dependents_may_launch();
    grid_dependency_wait();
    if (r < 0) {
        choose_slices(a, rows);
        return;
    }
    __nv_bfloat16 *scaled = a.scaled ? a.scaled + (int64_t)r * a.Kp : nullptr;
    if (r >= rows) {
        // up to the next block of the contraction: zeros that product 3 reads (U has its own)
        if (scaled && r < (rows + kBlockK - 1) / kBlockK * kBlockK)
            for (int k = threadIdx.x; k < a.K; k += kRowThreads) {
                scaled[k] = __float2bfloat16_rn(0.f);
                if (a.second) scaled[a.second + k] = __float2bfloat16_rn(0.f);
            }
        return;
    }
    const int label = info.x;
    const float row_c = __int_as_float(info.z);
    const bool bad = label < 0 || label >= a.V;
    const float4 *part = a.part + (size_t)r * a.chunks;
    float4 mine[2];                                             // this thread's first two chunks
    float m = kNoRef;
    const float acc = bad ? __int_as_float(0x7fffffff) : a.picked[r];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int t = j * kRowThreads + threadIdx.x;
        mine[j] = t < a.chunks ? part[t] : make_float4(kNoRef, 0.f, 0.f, 0.f);
        m = fmaxf(m, mine[j].x);
    }
    for (int t = threadIdx.x + 2 * kRowThreads; t < a.chunks; t += kRowThreads) m = fmaxf(m, part[t].x);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
    if (lane == 0) red[0][warp] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kRowThreads / 32; ++w) m = fmaxf(m, red[0][w]);
    float s = 0.f, sr = 0.f;                                    // sums of U and of the rounded U
    for (int t = threadIdx.x; t < a.chunks; t += kRowThreads) {
        const float4 p = t < kRowThreads ? mine[0] : t < 2 * kRowThreads ? mine[1] : part[t];
        // (2^-128 is no normal number, but 2^64 times it counts beside a largest value of 2^-64: in two steps)
        const float f = ex2(0.5f * (p.x - m));
        s = fmaf(p.y * f, f, s);
        sr = fmaf(p.z * f, f, sr);
        if (p.x != m && a.u) {
            // (16-byte pieces of 8 columns; the columns behind V are not used)
            uint4 *u = reinterpret_cast<uint4 *>(a.u + (int64_t)r * a.Vp + (int64_t)t * kChunk);
            const int64_t left = a.Vp - (int64_t)t * kChunk;
            for (int j = 0; j < kChunk / 8 && j * 8 < left; ++j) {
                uint4 v = u[j];
                uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = pack2(low(w[e]) * f * f, high(w[e]) * f * f);
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
    if (threadIdx.x == 0) {
        a.nll[row] = ((m - acc * row_c) + l2s) * kLn2;
        if (a.lse) a.lse[row] = fmaf(m + l2s, kLn2, __int_as_float(info.w));
        if (bad && a.status) atomicOr(a.status, PPO_DEV_BAD_TOKEN);
    }
    if (!a.u) return;
    // U at the label, as product 1 stored it, less S
    float f = nan, c = nan;
    if (!bad) {
        const float ref = part[label / kChunk].x;
        const float step = ex2(0.5f * (ref - m)), u = __bfloat162float(__float2bfloat16_rn(ex2(fmaf(acc, row_c, -ref)))) * step * step;
        const float want = u - sr;
        const __nv_bfloat16 stored = __float2bfloat16_rn(want);
        const float got = __bfloat162float(stored);
        f = a.scale * a.inv_tau / ((a.denom ? *a.denom : (float)n_real) * sr);
        if (got != 0.f) f *= want / got;
        c = f * (want - got);
        if (threadIdx.x == 0) a.u[(int64_t)r * a.Vp + label] = stored;
    }
    if (threadIdx.x == 0) a.row_scale[r] = make_float2(f, c);
    if (!scaled) return;
    for (int k = threadIdx.x * 8; k < a.K; k += kRowThreads * 8) {
        if (k + 8 <= a.K) {
            const uint4 v = k < kRowThreads * 8 ? ahead[0] : k < 2 * kRowThreads * 8 ? ahead[1] : *reinterpret_cast<const uint4 *>(h + k);
            const uint32_t u[4] = {v.x, v.y, v.z, v.w};
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = pack2(low(u[e]) * f, high(u[e]) * f);
            *reinterpret_cast<uint4 *>(scaled + k) = make_uint4(w[0], w[1], w[2], w[3]);
            if (a.second) {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = pack2(left_over(low(u[e]) * f, low(w[e])), left_over(high(u[e]) * f, high(w[e])));
                *reinterpret_cast<uint4 *>(scaled + a.second + k) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        } else {
            for (int e = k; e < a.K; ++e) {
                const float x = __bfloat162float(h[e]) * f;
                const __nv_bfloat16 y = __float2bfloat16_rn(x);
                scaled[e] = y;
                if (a.second) scaled[a.second + e] = __float2bfloat16_rn(left_over(x, __bfloat162float(y)));
            }
        }
    }
}

template <int THREADS>
__device__ __forceinline__ void sum_loss(const RowArgs &a)
{
    __shared__ double red[32];
    double s = 0.0;
#pragma unroll 8
    for (int i = threadIdx.x; i < a.M; i += THREADS) s += (double)a.nll[i];
    s = block_sum<THREADS>(s, red);
    if (threadIdx.x == 0) {
        const int n = *a.n_real;
        *a.loss = n ? (float)(s / (a.denom ? (double)*a.denom : (double)n)) : 0.f;
        if (!n && a.status) atomicOr(a.status, PPO_DEV_EMPTY_MASK);
    }
}

constexpr int kLossThreads = 1024;
__global__ void __launch_bounds__(kLossThreads)
loss_kernel(const RowArgs a)
{
    grid_dependency_wait();
    sum_loss<kLossThreads>(a);
}

// the last launch of some calls with one piece: the loss beside the joining of product 2's slices
template <int MODE>
__global__ void __launch_bounds__(kJoinThreads)
tail_kernel(const RowArgs r, const Args a, int workers)
{
    grid_dependency_wait();
    if (blockIdx.x == 0) sum_loss<kJoinThreads>(r);
    else join_tiles<MODE>(a, workers, blockIdx.x - 1);
}

// ---------------------------------------------------------------- host side
constexpr int kPieceRows = 256;                                 // a piece is a multiple of this

// few rows: the mode of products 1 and 2 (product 3 has its rows along the contraction), and a H in two parts
static bool few(int M) { return M <= 64; }

struct Layout {
    int pieces, rows_max, chunks, Kp;
    int64_t Vp;
    size_t n_real, slices, order, info, w_mean, w_one, picked, row_scale, part, packed, scaled, u, parts, sums, bytes;
};

// Pieces of at most 8192 rows by default: at V = 50304 that is 824 MB of U, and the sums of dW, read and written once a
// piece, are under a tenth of the piece's traffic.
static Layout layout_of(int64_t M, int64_t K, int64_t V, int64_t piece_rows, bool dh, bool dw)
{
    Layout l;
    const int64_t asked = piece_rows > 0 ? piece_rows : 8192, most = asked < M ? asked : M;      // (any number may be asked for)
    l.pieces = (int)((M + most - 1) / most);
    const int64_t even = (M + l.pieces - 1) / l.pieces;
    l.rows_max = (int)((even + kPieceRows - 1) / kPieceRows * kPieceRows);
    l.pieces = (int)((M + l.rows_max - 1) / l.rows_max);
    l.chunks = (int)((V + kChunk - 1) / kChunk);
    // (rows of whole 128-byte lines: a row of a box that begins inside a line costs two requests)
    l.Kp = (int)((K + 63) / 64 * 64);
    l.Vp = (V + 63) / 64 * 64;
    size_t at = 0;
    const auto take = [&](size_t n) {
        const size_t here = at;
        at += align256(n);
        return here;
    };
    const bool grad = dh || dw;
    const size_t rows = (size_t)l.rows_max;
    l.n_real = take(4);
    l.slices = take(8);
    l.order = take((size_t)M * 4);
    l.info = take((size_t)M * sizeof(int4));
    l.w_mean = take((size_t)(K + 511) / 512 * 512 * 4);
    l.w_one = take((size_t)K * 4);
    l.picked = take(rows * 4);
    l.row_scale = take(rows * sizeof(float2));
    l.part = take(rows * (size_t)l.chunks * sizeof(float4));
    l.packed = take((size_t)M * l.Kp * 2);
    l.scaled = take(dw ? rows * l.Kp * 2 * (few((int)M) ? 2 : 1) : 0);
    l.u = take(grad ? rows * (size_t)l.Vp * 2 : 0);
    l.parts = take(!dh ? 0 : (size_t)2 * 4 * (M <= kBM ? kMaxSms * Shape<kSingle>::kTileFloats : kMaxSms / 2 * Shape<kWide>::kTileFloats));
    // (whole tiles, in either layout)
    const size_t up_k = (size_t)(K + 511) / 512 * 512, up_v = (size_t)(V + 511) / 512 * 512;
    l.sums = take(dw && l.pieces > 1 ? up_k * up_v * 4 : 0);
    l.bytes = at;
    return l;
}

static int sms_of_device(int *sms)
{
    int dev = 0;
    *sms = 148;
    PPO_RETURN_IF_CUDA(cudaGetDevice(&dev));
    PPO_RETURN_IF_CUDA(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev));
    if (*sms > kMaxSms) *sms = kMaxSms;
    return PPO_OK;
}

template <int MODE, bool A_MN, bool B_MN, int PRODUCT>
static int launch_product(const CUtensorMap &ma, const CUtensorMap &ma_all, const CUtensorMap &mb, const CUtensorMap &mo, const Args &a,
                          int sms, cudaStream_t s)
{
    constexpr bool PAIR = Shape<MODE>::kIsPair;
    auto kern = product_kernel<MODE, A_MN, B_MN, PRODUCT>;
    PPO_RETURN_IF_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<MODE>::kSmem));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(PAIR ? sms / 2 * 2 : sms));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Shape<MODE>::kSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = PAIR ? 2 : 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, kern, ma, ma_all, mb, mo, a);
    if (e != cudaSuccess) {   // the first attribute is not accepted in this context: ordinary launch (same results, no overlap)
        (void)cudaGetLastError();
        cfg.attrs = attr + 1;
        cfg.numAttrs = PAIR ? 1 : 0;
        e = cudaLaunchKernelEx(&cfg, kern, ma, ma_all, mb, mo, a);
    }
    PPO_RETURN_IF_CUDA(e);
    return PPO_OK;
}

// the three products of a piece
struct Maps {
    CUtensorMap packed, h, w1, w2, u_out, u2, u3, scaled, dw;
};

template <int MODE>
static int launch_hidden(const Maps &m, const Args &a2, bool vk, int sms, cudaStream_t s)
{
    const int rc = vk ? launch_product<MODE, false, true, kHidden>(m.u2, m.u2, m.w2, m.u2, a2, sms, s)
                      : launch_product<MODE, false, false, kHidden>(m.u2, m.u2, m.w2, m.u2, a2, sms, s);
    return rc;
}

// what follows product 2, or (last: with the loss) product 3
template <int MODE>
static int launch_join(const RowArgs &r, const Args &a2, bool last, int sms, cudaStream_t s)
{
    const int workers = Shape<MODE>::kIsPair ? sms / 2 : sms;
    const unsigned blocks = (unsigned)((workers - 1) * join_blocks<MODE>());
    if (last) PPO_RETURN_IF_CUDA(launch_dependent(tail_kernel<MODE>, dim3(1 + blocks), dim3(kJoinThreads), 0, s, r, a2, workers));
    else PPO_RETURN_IF_CUDA(launch_dependent(join_kernel<MODE>, dim3(blocks), dim3(kJoinThreads), 0, s, a2, workers));
    return PPO_OK;
}

template <int MODE>
static int launch_weight(const Maps &m, const Args &a3, bool vk, int sms, cudaStream_t s)
{
    return vk ? launch_product<MODE, true, true, kWeight>(m.u3, m.u3, m.scaled, m.dw, a3, sms, s)
              : launch_product<MODE, true, true, kWeight>(m.scaled, m.scaled, m.u3, m.dw, a3, sms, s);
}

// Wide tiles where they are half as many, the contraction is at least 64 blocks long (their epilogue, 6000 cycles for two
// accumulators, has to be small against 1024 a block) and the pairs get two tiles or more each (6912 x 4096 x 50304, W [V, K]: dH
// 1973 us against 2049, dW 2017 against 2077; 1792 rows, whose 56 wide tiles are all cut: dH 598 against 544). (dW of W [K, V] at V = 50304,
// 197 tiles of 256, is not among them.)
static bool wide(int64_t m, int64_t n, int64_t contraction, int sms)
{
    return (n + 255) / 256 % 2 == 0 && contraction >= 64 * kBlockK && (m + 255) / 256 * ((n + 511) / 512) >= sms;
}

template <int MODE>
static void set_shape(RowArgs &r, const Args &a2, int sms)
{
    using S = Shape<MODE>;
    r.tile_m = S::kM;
    r.n_tiles = (a2.dim_n + S::kN - 1) / S::kN;
    r.workers = S::kIsPair ? sms / 2 : sms;
    r.kbs = (a2.dim_k + kBlockK - 1) / kBlockK;
}

static int launch_piece(const Maps &m, RowArgs r, const Args &a1, Args a2, Args a3, bool single, bool vk, bool dh, bool dw, bool only,
                        int sms, cudaStream_t s)
{
    int rc;
    const bool small = few(a1.M);
    if (small)
        rc = vk ? launch_product<kSmall, false, false, kLogits>(m.packed, m.h, m.w1, m.u_out, a1, sms, s)
                : launch_product<kSmall, false, true, kLogits>(m.packed, m.h, m.w1, m.u_out, a1, sms, s);
    else if (single)
        rc = vk ? launch_product<kSingle, false, false, kLogits>(m.packed, m.h, m.w1, m.u_out, a1, sms, s)
                : launch_product<kSingle, false, true, kLogits>(m.packed, m.h, m.w1, m.u_out, a1, sms, s);
    else
        rc = vk ? launch_product<kPair, false, false, kLogits>(m.packed, m.h, m.w1, m.u_out, a1, sms, s)
                : launch_product<kPair, false, true, kLogits>(m.packed, m.h, m.w1, m.u_out, a1, sms, s);
    if (rc) return rc;
    const bool wide_hidden = !single && wide(a2.dim_m, a2.dim_n, a2.dim_k, sms);
    if (single) set_shape<kSingle>(r, a2, sms);
    else if (wide_hidden) set_shape<kWide>(r, a2, sms);
    else set_shape<kPair>(r, a2, sms);
    PPO_RETURN_IF_CUDA(launch_dependent(row_kernel, dim3(1 + (unsigned)r.rows_max), dim3(kRowThreads), 0, s, r));
    const auto join = [&](bool last) {
        return wide_hidden ? launch_join<kWide>(r, a2, last, sms, s) : small ? launch_join<kSmall>(r, a2, last, sms, s)
               : single    ? launch_join<kSingle>(r, a2, last, sms, s) : launch_join<kPair>(r, a2, last, sms, s);
    };
    if (dh) {
        if (wide_hidden) {
            a2.gm = 12;
            a2.gn = 6;
        }
        rc = wide_hidden ? launch_hidden<kWide>(m, a2, vk, sms, s) : small ? launch_hidden<kSmall>(m, a2, vk, sms, s)
             : single    ? launch_hidden<kSingle>(m, a2, vk, sms, s) : launch_hidden<kPair>(m, a2, vk, sms, s);
        if (!rc && !only) rc = join(false);
        if (rc) return rc;
    }
    if (dw) {
        // (the number of pieces does not change the mode: their sums lie in its order)
        if (!single && wide(a3.dim_m, a3.dim_n, a3.dim_k, sms)) {
            a3.gm = 12;
            a3.gn = 6;
            rc = launch_weight<kWide>(m, a3, vk, sms, s);
        } else {
            rc = small ? launch_weight<kTwice>(m, a3, vk, sms, s) : single ? launch_weight<kSingle>(m, a3, vk, sms, s) : launch_weight<kPair>(m, a3, vk, sms, s);
        }
        if (rc) return rc;
    }
    return dh && only ? join(true) : PPO_OK;
}

constexpr int64_t kLimit = ((int64_t)1 << 31) - 16384;

static bool sizes_ok(int64_t M, int64_t K, int64_t V, int64_t piece_rows)
{
    return M > 0 && K > 0 && V > 0 && M < kLimit && K < kLimit && V < kLimit && piece_rows >= 0 &&
           ((K + 255) / 256) * ((V + 255) / 256) < ((int64_t)1 << 27) && ((M + 255) / 256) * ((V + 255) / 256) < ((int64_t)1 << 27);
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
        reinterpret_cast<uintptr_t>(dH) % 2 || reinterpret_cast<uintptr_t>(dW) % 2 || reinterpret_cast<uintptr_t>(labels) % 4 ||
        reinterpret_cast<uintptr_t>(loss) % 4 || reinterpret_cast<uintptr_t>(nll) % 4 || reinterpret_cast<uintptr_t>(lse) % 4 ||
        reinterpret_cast<uintptr_t>(denom) % 4 || reinterpret_cast<uintptr_t>(workspace) % 256)
        return PPO_ERR_ALIGN;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    int *status = workspace ? &ws_header(workspace)->status : nullptr;
    if (M == 0) {
        PPO_RETURN_IF_CUDA(cudaMemsetAsync(loss, 0, 4, s));
        if (dW) PPO_RETURN_IF_CUDA(cudaMemset2DAsync(dW, (size_t)lddw * 2, 0, (size_t)w_inner * 2, (size_t)w_outer, s));
        return PPO_OK;
    }
    int sms = 0;
    int rc = sms_of_device(&sms);
    if (rc) return rc;
    const Layout l = layout_of(M, K, V, piece_rows, dH != nullptr, dW != nullptr);
    unsigned char *mem = reinterpret_cast<unsigned char *>(scratch);
    const bool grad = dH || dW;

    RowArgs r = {};
    r.H = reinterpret_cast<const __nv_bfloat16 *>(H);
    r.ldh = ldh; r.lddh = lddh; r.M = (int)M; r.K = (int)K; r.V = (int)V; r.Kp = l.Kp;
    r.labels = labels; r.mask = mask; r.ignore_id = ignore_id;
    r.c = 1.4426950408889634 / (double)temperature;
    r.inv_tau = 1.f / temperature; r.scale = scale; r.denom = denom;
    r.n_real = reinterpret_cast<int *>(mem + l.n_real);
    r.order = reinterpret_cast<int32_t *>(mem + l.order);
    r.W = reinterpret_cast<const __nv_bfloat16 *>(W); r.ldw = ldw; r.vk = vk;
    r.w_mean = reinterpret_cast<float *>(mem + l.w_mean);
    r.w_one = reinterpret_cast<float *>(mem + l.w_one);
    r.info = reinterpret_cast<int4 *>(mem + l.info);
    r.in_place = ldh % 64 == 0 && reinterpret_cast<uintptr_t>(H) % 128 == 0;
    r.packed = reinterpret_cast<__nv_bfloat16 *>(mem + l.packed);
    r.scaled = dW ? reinterpret_cast<__nv_bfloat16 *>(mem + l.scaled) : nullptr;
    const bool twice = few((int)M);                              // (product 3's mode: see there)
    r.second = twice ? (int64_t)l.rows_max * l.Kp : 0;
    r.u = grad ? reinterpret_cast<__nv_bfloat16 *>(mem + l.u) : nullptr;
    r.Vp = l.Vp;
    r.picked = reinterpret_cast<float *>(mem + l.picked);
    r.row_scale = reinterpret_cast<float2 *>(mem + l.row_scale);
    r.part = reinterpret_cast<float4 *>(mem + l.part);
    r.chunks = l.chunks; r.rows_max = l.rows_max;
    r.loss = loss; r.nll = nll; r.lse = lse; r.dH = reinterpret_cast<__nv_bfloat16 *>(dH);
    r.status = status;

    Maps m = {};
    const int rows_a = few((int)M) ? 64 : kBM;                  // rows of A that a load brings
    const int rows_b = Shape<kPair>::kRowsB;                    // a block's share of B, stored by rows
    if ((rc = make_map_pitch(&m.packed, r.packed, (uint64_t)K, (uint64_t)M, (uint64_t)l.Kp, rows_a))) return rc;
    if ((rc = make_map_pitch(&m.h, H, (uint64_t)K, (uint64_t)M, (uint64_t)ldh, rows_a))) return rc;
    // product 1 takes W with the vocabulary as the result's columns, product 2 with the hidden size
    if ((rc = make_map_pitch(&m.w1, W, (uint64_t)w_inner, (uint64_t)w_outer, (uint64_t)ldw, vk ? rows_b : 64))) return rc;
    if ((rc = make_map_pitch(&m.w2, W, (uint64_t)w_inner, (uint64_t)w_outer, (uint64_t)ldw, vk ? 64 : rows_b))) return rc;
    if (grad) {
        if ((rc = make_map_pitch(&m.u_out, r.u, (uint64_t)V, (uint64_t)l.rows_max, (uint64_t)l.Vp, 32))) return rc;
        if ((rc = make_map_pitch(&m.u2, r.u, (uint64_t)V, (uint64_t)l.rows_max, (uint64_t)l.Vp, rows_a))) return rc;
        if ((rc = make_map_pitch(&m.u3, r.u, (uint64_t)V, (uint64_t)l.rows_max, (uint64_t)l.Vp, 64))) return rc;
    }

    Args a = {};
    a.n_real = r.n_real; a.M = (int)M; a.rows_max = l.rows_max; a.status = status;
    a.order = r.order; a.info = r.info; a.in_place = r.in_place;
    a.picked = r.picked; a.part = r.part; a.chunks = l.chunks; a.store = grad;
    a.row_scale = r.row_scale;
    Args a1 = a, a2 = a, a3 = a;
    // (blocks of gm x gn = 72 tiles, which as many pairs work on at a time, near square in elements: they share panels through L2)
    a1.dim_m = l.rows_max; a1.dim_n = (int)V; a1.dim_k = (int)K; a1.gm = 9; a1.gn = 8;
    a2.dim_m = l.rows_max; a2.dim_n = (int)K; a2.dim_k = (int)V; a2.gm = 9; a2.gn = 8;
    a2.out = r.dH; a2.ldo = lddh; a2.w_mean = r.w_mean;
    a2.slices = r.slices = reinterpret_cast<int2 *>(mem + l.slices);
    a2.scratch = reinterpret_cast<float *>(mem + l.parts);
    a3.dim_m = (int)w_outer; a3.dim_n = (int)w_inner; a3.dim_k = l.rows_max; a3.gm = 8; a3.gn = 9;
    a3.out = reinterpret_cast<__nv_bfloat16 *>(dW); a3.ldo = lddw;
    a3.scratch = reinterpret_cast<float *>(mem + l.sums);
    a3.vk = vk; a3.second = l.rows_max;
    if (dW) {
        if ((rc = make_map_pitch(&m.scaled, r.scaled, (uint64_t)K, (uint64_t)l.rows_max * (twice ? 2 : 1), (uint64_t)l.Kp, 64))) return rc;
        if (reinterpret_cast<uintptr_t>(dW) % 16 == 0 && lddw % 8 == 0 && lddw < ((int64_t)1 << 38)) {
            // (a box is clipped in units of 16 bytes: it would write zeros behind a row whose end is none)
            a3.bulk_cols = w_inner % 8 ? (int)w_inner : 0x7fffffff;
            if ((rc = make_map_pitch(&m.dw, dW, (uint64_t)w_inner, (uint64_t)w_outer, (uint64_t)lddw, 32))) return rc;
        }
    }

    // (the first launch waits for all work before the call, the others for the one before them)
    order_kernel<<<1 + (unsigned)((K + kMeanPer - 1) / kMeanPer), kOrderThreads, 0, s>>>(r);
    if ((rc = launch_status())) return rc;
    PPO_RETURN_IF_CUDA(launch_dependent(pack_kernel, dim3((unsigned)M), dim3(kRowThreads), 0, s, r));
    // The loss and the joining in one launch at the end, unless dW takes the slices out of L2 before that (100 x 20000 x 1032: 75 us in
    // two launches, 70 in one; 300 x 50304 x 1032: 171 and
    // 176)
    const bool tail = l.pieces == 1 && K * V <= 1 << 25;
    for (int p = 0; p < l.pieces; ++p) {
        r.row0 = a1.row0 = a2.row0 = a3.row0 = p * l.rows_max;
        rc = launch_piece(m, r, a1, a2, a3, M <= kBM, vk, dH != nullptr, dW != nullptr, tail, sms, s);
        if (rc) return rc;
    }
    if (!dH || !tail) PPO_RETURN_IF_CUDA(launch_dependent(loss_kernel, dim3(1), dim3(kLossThreads), 0, s, r));
    return PPO_OK;
}
