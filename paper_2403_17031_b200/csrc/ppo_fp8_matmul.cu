// Product of two block-scaled 8-bit matrices (ppo_fp8_matmul):
//     C[m, n] = sum over blocks b of 128 along K of  sa[b, m] * sb[b, n] * sum_{k in b} A[m, k] B[n, k]
// A [M, K], B [N, K] e4m3, both K-contiguous; sa one scale per row and block, sb one per 128 rows (or per row) and
// block. The tensor core forms the inner sums (exact products, fp32 accumulation) into tensor memory, one fresh
// accumulator per block of K; the epilogue warps multiply each by its scales and add it to fp32 registers while the
// tensor core is already on the next block.
//
// Narrow kernel (few rows of A): the weight B supplies the 128 lanes of the accumulator tile and the rows of A its
// columns, so that a tile never holds more than 16 idle rows and the stream of B, which bounds the call, is read by
// full 128 x 128 boxes. K is split over a cluster of blocks when there are too few tiles to occupy the SMs; the
// partial tiles are joined through distributed shared memory in rank order, so results do not depend on timing.
// 1 x 50304 x 4096 (206 MB of weight): 35.6 us = 5.8 TB/s with rings of three stages, so that four blocks fit on an SM and all
// 393 tiles are under way at once (four stages and three blocks: 36.9 us, six and two: 43 us).
#include <cooperative_groups.h>

#include "ppo_tcgen05.cuh"

namespace ppo {
namespace fp8 {

namespace cg = cooperative_groups;
using namespace tc;

constexpr int kBlockK = 128;           // one scale block, one 128-byte swizzle row

struct Args {
    int M, N, kb_total;
    const float *sa;                   // [kb_total, M]
    const float *sb;                   // [ceil(N/128), kb_total], or [kb_total, N] with per_row
    int per_row;
    void *out;
    int64_t ldc;
    int out_f32;
    int m_tiles, n_tiles;
    int *status;
};

// PPO_TEST_WITHHOLD_FP8 (never defined in the product build): a test build in which, from the third block of K on (the second group of
// scales), 1: products, 2: scales or 3: released accumulators are never announced, so that the waits for them run out.
#ifndef PPO_TEST_WITHHOLD_FP8
#define PPO_TEST_WITHHOLD_FP8 0
#endif
enum Withheld { kProducts = 1, kScaleGroups = 2, kReleases = 3 };
__device__ __forceinline__ bool withheld(Withheld what, int done, int allowed) { return PPO_TEST_WITHHOLD_FP8 == what && done >= allowed; }

// A wait that is skipped once one has run out: the block then reaches its end quickly, with the same control flow. Whoever has given
// up announces nothing any more, so that the others' waits run out too instead of going on with what nobody computed, and an
// epilogue warp that has given up stores NaN: without a status word that is the only sign.
__device__ __forceinline__ void wait_alive(bool &alive, unsigned long long *bar, uint32_t parity, int *status)
{
    if (alive) alive = wait(bar, parity, status);
}

constexpr int kNarrowBufs = 2, kNarrowThreads = 192;

// ST: stages of the ring
template <int MT, int ST>
struct NarrowSmem {
    unsigned long long full[ST], empty[ST], tmem_full[kNarrowBufs], tmem_empty[kNarrowBufs];
    uint32_t tmem_base;
    int issued;                               // blocks of K whose products were issued
    float4 scale[4][kNarrowBufs][MT / 4];     // per epilogue warp: the columns' factors of a block of K
};

template <int MT> __host__ __device__ constexpr int narrow_stage_bytes() { return (128 + MT) * kBlockK; }
// accumulator columns: a power of two, at least 32
template <int MT> __host__ __device__ constexpr uint32_t narrow_columns() { return kNarrowBufs * MT < 32 ? 32 : kNarrowBufs * MT; }

// four neighbouring results of row m; vec: all of them inside, at an aligned address
__device__ __forceinline__ void store4(const Args &a, int m, int n, const float4 &v, bool vec)
{
    if (m >= a.M) return;
    const float x[4] = {v.x, v.y, v.z, v.w};
    if (a.out_f32) {
        float *to = reinterpret_cast<float *>(a.out) + (int64_t)m * a.ldc + n;
        if (vec) *reinterpret_cast<float4 *>(to) = v;
        else
            for (int e = 0; e < 4 && n + e < a.N; ++e) to[e] = x[e];
    } else {
        __nv_bfloat16 *to = reinterpret_cast<__nv_bfloat16 *>(a.out) + (int64_t)m * a.ldc + n;
        if (vec) {
            const __nv_bfloat162 lo = __floats2bfloat162_rn(x[0], x[1]), hi = __floats2bfloat162_rn(x[2], x[3]);
            *reinterpret_cast<uint2 *>(to) = make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
        } else
            for (int e = 0; e < 4 && n + e < a.N; ++e) to[e] = __float2bfloat16_rn(x[e]);
    }
}

template <int MT, int ST>
__global__ void __launch_bounds__(kNarrowThreads)
narrow_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const Args a, int split)
{
    constexpr int kStage = narrow_stage_bytes<MT>();
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ NarrowSmem<MT, ST> sm;
    unsigned char *ring = smem_raw + ((1024u - (saddr(smem_raw) & 1023u)) & 1023u);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = blockIdx.x % split, tile = blockIdx.x / split;
    const int m0 = (tile % a.m_tiles) * MT, n0 = (tile / a.m_tiles) * 128;
    const int kb0 = (int)((int64_t)a.kb_total * rank / split), kb1 = (int)((int64_t)a.kb_total * (rank + 1) / split);

    if (threadIdx.x == 0) {
        for (int s = 0; s < ST; ++s) {
            barrier_init(&sm.full[s], 1);
            barrier_init(&sm.empty[s], 1);
        }
        for (int b = 0; b < kNarrowBufs; ++b) {
            barrier_init(&sm.tmem_full[b], 1);
            barrier_init(&sm.tmem_empty[b], 4);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(&sm.tmem_base, narrow_columns<MT>());
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = sm.tmem_base;
    float acc[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[j] = 0.f;

    if (warp == 0) {
        if (lane == 0) {
            bool alive = true;
            int issued = 0;
            for (int kb = kb0; kb < kb1; ++kb, ++issued) {
                const int s = issued % ST;
                if (issued >= ST) wait_alive(alive, &sm.empty[s], ((issued / ST) - 1) & 1, a.status);
                if (!alive) break;
                unsigned char *stage = ring + (size_t)s * kStage;
                barrier_expect_tx(&sm.full[s], (uint32_t)kStage);
                tma_load_2d(stage, &map_b, kb * kBlockK, n0, &sm.full[s]);
                tma_load_2d(stage + 128 * kBlockK, &map_a, kb * kBlockK, m0, &sm.full[s]);
            }
            // copies in flight land before the block may end
            for (int i = issued > ST ? issued - ST : 0; i < issued; ++i)
                wait(&sm.full[i % ST], (i / ST) & 1, a.status);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr uint32_t idesc = instr_desc_e4m3(128, MT);
            bool alive = true;
            int i = 0;
            for (; i < kb1 - kb0 && !withheld(kProducts, i, 2); ++i) {
                const int s = i % ST, buf = i % kNarrowBufs;
                if (i >= kNarrowBufs) wait_alive(alive, &sm.tmem_empty[buf], ((i / kNarrowBufs) - 1) & 1, a.status);
                wait_alive(alive, &sm.full[s], (i / ST) & 1, a.status);
                if (!alive) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t b_addr = saddr(ring + (size_t)s * kStage), a_addr = b_addr + 128 * kBlockK;
#pragma unroll
                for (int kk = 0; kk < kBlockK / 32; ++kk)
                    mma_f8(tmem_base + buf * MT, smem_desc(b_addr + kk * 32, 16, 1024), smem_desc(a_addr + kk * 32, 16, 1024),
                           idesc, kk ? 1u : 0u);
                commit(&sm.empty[s]);
                commit(&sm.tmem_full[buf]);
            }
            sm.issued = i;
            // every product has ended before tensor memory is freed
            if (i > 0) wait(&sm.tmem_full[(i - 1) % kNarrowBufs], ((i - 1) / kNarrowBufs) & 1, a.status);
        }
        __syncwarp();
    } else {
        // lane (warp & 3) * 32 + lane of the accumulator is row n of B
        const int q = warp & 3, n = n0 + q * 32 + lane;
        bool alive = true;
        constexpr int J = (MT + 31) / 32;
        float next_sa[J], next_sb = 0.f;               // the next block's scales, loaded one block ahead
        auto fetch = [&](int kb) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int m = m0 + j * 32 + lane;
                next_sa[j] = (MT >= 32 || lane < MT) && m < a.M ? a.sa[(int64_t)kb * a.M + m] : 0.f;
            }
            next_sb = n >= a.N ? 0.f : a.per_row ? a.sb[(int64_t)kb * a.N + n] : a.sb[(int64_t)(n0 / 128) * a.kb_total + kb];
        };
        if (kb0 < kb1) fetch(kb0);
        for (int i = 0; i < kb1 - kb0; ++i) {
            const int kb = kb0 + i, buf = i % kNarrowBufs;
            float *sc = reinterpret_cast<float *>(sm.scale[q][buf]);
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (MT >= 32 || lane < MT) sc[j * 32 + lane] = next_sa[j];
            const float sb = next_sb;
            if (kb + 1 < kb1) fetch(kb + 1);
            wait_alive(alive, &sm.tmem_full[buf], (i / kNarrowBufs) & 1, a.status);
            __syncwarp();
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t taddr = tmem_base + buf * MT + ((uint32_t)(q * 32) << 16);
#pragma unroll
            for (int g = 0; g < MT / 16; ++g) {
                uint32_t r[16];
                tmem_ld16(taddr + g * 16, r);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                if (g == MT / 16 - 1) {
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0 && alive && !withheld(kReleases, i, 2)) barrier_arrive(&sm.tmem_empty[buf]);
                }
#pragma unroll
                for (int j4 = 0; j4 < 4; ++j4) {
                    const float4 f = sm.scale[q][buf][g * 4 + j4];
                    float *d = acc + g * 16 + j4 * 4;
                    const uint32_t *p = r + j4 * 4;
                    d[0] = fmaf(__uint_as_float(p[0]), f.x * sb, d[0]);
                    d[1] = fmaf(__uint_as_float(p[1]), f.y * sb, d[1]);
                    d[2] = fmaf(__uint_as_float(p[2]), f.z * sb, d[2]);
                    d[3] = fmaf(__uint_as_float(p[3]), f.w * sb, d[3]);
                }
            }
        }
        if (!alive) {
#pragma unroll
            for (int j = 0; j < MT; ++j) acc[j] = __uint_as_float(0x7fffffffu);
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        tmem_free(tmem_base, narrow_columns<MT>());
    }
    // Every copy has landed and every product is done: the ring is free for the join. Nobody has waited for the last arrivals on
    // its barriers, though, and the block must not end before them: a lane for each. (Beside the stores: one after the other and
    // before the barrier above, these waits took 64 x 4096 x 8192 from 13.7 to 14.6 us.)
    const auto drain = [&] {
        const int i = sm.issued - 1 - lane;
        if (warp == 1 && lane < ST && i >= 0) wait(&sm.empty[i % ST], (i / ST) & 1, a.status);
    };
    const int q = warp & 3, nl = q * 32 + lane, n = n0 + nl;
    if (split > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        float *part = reinterpret_cast<float *>(ring);             // [MT][128]
        if (warp >= 2) {
#pragma unroll
            for (int j = 0; j < MT; ++j) part[j * 128 + nl] = acc[j];
        }
        cluster.sync();
        drain();
        if (warp >= 2) {
            // columns rank, rank + split, ... of the tile; a warp takes every fourth of them, a lane four rows of B, and
            // the remote loads of two columns are under way together
            const int r4 = lane * 4;
            const bool vec = n0 + 128 <= a.N && (reinterpret_cast<uintptr_t>(a.out) & 15u) == 0 && (a.ldc & 3) == 0;
            for (int j0 = rank + q * split; j0 < MT; j0 += 8 * split) {
                const int j1 = j0 + 4 * split;
                float4 v0 = make_float4(0.f, 0.f, 0.f, 0.f), v1 = v0;
                for (int r = 0; r < split; ++r) {
                    const float *from = cluster.map_shared_rank(part, r);
                    const float4 x0 = *reinterpret_cast<const float4 *>(from + j0 * 128 + r4);
                    const float4 x1 = *reinterpret_cast<const float4 *>(from + (j1 < MT ? j1 : j0) * 128 + r4);
                    v0.x += x0.x; v0.y += x0.y; v0.z += x0.z; v0.w += x0.w;
                    v1.x += x1.x; v1.y += x1.y; v1.z += x1.z; v1.w += x1.w;
                }
                store4(a, m0 + j0, n0 + r4, v0, vec);
                if (j1 < MT) store4(a, m0 + j1, n0 + r4, v1, vec);
            }
        }
        cluster.sync();
        return;
    }
    drain();
    if (warp >= 2 && n < a.N) {
#pragma unroll
        for (int j = 0; j < MT; ++j) {
            const int m = m0 + j;
            if (m < a.M) {
                if (a.out_f32) reinterpret_cast<float *>(a.out)[(int64_t)m * a.ldc + n] = acc[j];
                else reinterpret_cast<__nv_bfloat16 *>(a.out)[(int64_t)m * a.ldc + n] = __float2bfloat16_rn(acc[j]);
            }
        }
    }
}

// blocks that fit on the SMs at once, by their shared memory (73, 81 and 97 KB with four stages)
template <int MT> constexpr int narrow_places() { return (MT == 16 ? 3 : 2) * 148; }

template <int MT, int ST>
static int launch_narrow_stages(const Args &a, const CUtensorMap &ma, const CUtensorMap &mb, int split, cudaStream_t s)
{
    const size_t smem = (size_t)ST * narrow_stage_bytes<MT>() + 1024;
    PPO_RETURN_IF_CUDA(cudaFuncSetAttribute(narrow_kernel<MT, ST>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.m_tiles * a.n_tiles * split));
    cfg.blockDim = dim3(kNarrowThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = split > 1 ? 1 : 0;
    PPO_RETURN_IF_CUDA(cudaLaunchKernelEx(&cfg, narrow_kernel<MT, ST>, ma, mb, a, split));
    return PPO_OK;
}

template <int MT>
static int launch_narrow(Args a, const void *A, int64_t lda, const void *B, int64_t ldb, int64_t K, cudaStream_t s)
{
    CUtensorMap ma, mb;
    int rc = make_map_8bit(&ma, A, (uint64_t)K, (uint64_t)a.M, (uint64_t)lda, MT);
    if (rc) return rc;
    rc = make_map_8bit(&mb, B, (uint64_t)K, (uint64_t)a.N, (uint64_t)ldb, 128);
    if (rc) return rc;
    a.m_tiles = (a.M + MT - 1) / MT;
    a.n_tiles = (a.N + 127) / 128;
    const int64_t tiles = (int64_t)a.m_tiles * a.n_tiles;
    // blocks of a tile's cluster: as many as fit on the SMs at once, each with two blocks of K or more
    int split = 1;
    while (split < 8 && tiles * split * 2 <= narrow_places<MT>() && a.kb_total >= 4 * split) split *= 2;
    if (tiles * split >= ((int64_t)1 << 31)) return PPO_ERR_SHAPE;
    // Tiles of 16 and 32 columns: three stages once the SMs hold more than two blocks each, so that another fits (1 x 50304 x
    // 4096: 35.6 instead of 36.9 us, 32 x 50304 x 4096: 40.5 instead of 51, 32 x 38000 x 4096: 32 instead of 52), else four
    // (4 x 16384 x 4096: 16.2 instead of 16.5 us)
    if constexpr (MT <= 32)
        if (tiles * split > 2 * 148) return launch_narrow_stages<MT, 3>(a, ma, mb, split, s);
    return launch_narrow_stages<MT, 4>(a, ma, mb, split, s);
}

// ---------------------------------------------------------------- wide kernel
// Rows of A are the lanes of the accumulator tile, 256 rows of B its columns. Two blocks on two SMs work as a pair on a
// 256 x 256 tile: one matrix instruction spans both tensor cores, each block loads its 128 rows of A and 128 of the 256
// rows of B and keeps 128 result rows. One persistent pair per two SMs, 768 threads a block:
//   warp 0      TMA producer (4 stages of 32 KB)
//   warp 1      scales, a group of blocks of K ahead of the epilogue (their latency is several blocks of K)
//   warps 4-7   of the leader: MMA issuers, one for each of four accumulators (half of the columns, one block of K)
//   warps 8-23  epilogue: warp (q, c) owns lanes 32 q .. and columns 64 c .., i.e. a thread holds 64 results of one row
//               and needs one factor sa * sb per block of K; the join is a packed fp32 multiply-add per two elements
// Bounds: with few tiles the hand-over of accumulators (from the end of a product to the start of the next one into the
// same accumulator lie about 1200 cycles of commits, barrier waits, which cost 100 to 200 cycles each even when they are
// over, fences and reads; two accumulators per half hide half of it: 0.52 us per block of K and tile); with many, the
// board's power limit: at 27136 x 50304 x 4096 a block of K takes 925 cycles, but the clock falls to 1.35 GHz. Compared
// under that load: blocks alone on 128 x 256 tiles 7.3 ms, pairs 6.0 to 6.4 ms; 256 x 192 tiles, whose accumulators can be released
// before anything is multiplied, 6.6 ms; one issuer instead of four 9 ms; 256-column accumulators 6.6 ms.
constexpr int kBM = 128, kBN = 256, kPairM = 2 * kBM, kWideStages = 4, kWideThreads = 768;
constexpr int kWideA = kBM * kBlockK, kWideB = kBN / 2 * kBlockK, kWideStage = kWideA + kWideB;   // a block's halves of A and B
constexpr int kStageOut = 32 * 128;        // per epilogue warp: 32 rows x 128 bytes
constexpr int kEpiWarps = 4 * (kBN / 64);
// blocks of K whose scales are handed over together (two groups in flight), and floats of one block: sa[128], sb (those of
// the two 128-row blocks of B, or of each row)
template <bool PER_ROW> struct Scales {
    static constexpr int kGroup = PER_ROW ? 4 : 16, kFloats = kBM + (PER_ROW ? kBN : 4), kBytes = 2 * kGroup * kFloats * 4;
};
constexpr int kScaleBytes = Scales<false>::kBytes > Scales<true>::kBytes ? Scales<false>::kBytes : Scales<true>::kBytes;
constexpr int kWideSmem = kWideStages * kWideStage + kEpiWarps * kStageOut + kScaleBytes + 1024;
static_assert(kWideSmem <= 232448 - 1024, "shared memory of a block");
static_assert(kWideThreads == (8 + kEpiWarps) * 32 && kWideStage % 1024 == 0 && kWideA % 1024 == 0, "layout");

struct WideSmem {
    unsigned long long full[kWideStages], empty[kWideStages], tmem_full[2][2];   // [half][accumulator]
    unsigned long long scale_full[2], scale_empty[2];
    unsigned long long pair_empty[2][2];   // the leader's: both blocks' epilogues have read the accumulator
    unsigned long long nobody[2];          // takes the arrivals of warps that have given up
    uint32_t tmem_base;
};

// The pairs take tiles 0 .. n_whole in turn, whole. With `share` > 0 the other tiles, too few for all pairs, are cut along
// K: end to end they are n_rest * kb_total blocks of K, of which pair c takes share, from c * share on. Such a pair leaves
// its sums of a tile in the scratch buffer (at most two tiles), and join_kernel adds them up in the order of the pairs.
struct WideArgs {
    Args a;
    int gm, gn, n_whole, n_rest, share;
    // Bulk stores take the boxes that end at or before this column: none where rows of C are not 16-byte aligned, those inside N where
    // N is not a multiple of 16 bytes (a box is clipped in units of 16 bytes: it would write zeros behind N), else all.
    int bulk_cols;
    float *scratch;
};

constexpr int kTileFloats = kPairM * kBN;

struct Piece {
    int u, kb0, kb1;      // tile, blocks of K
    int part;             // -1: whole; else which of the pair's sums in the scratch buffer
    int u_next, r, r_end;
    __device__ __forceinline__ void init(const WideArgs &w, int pair, int kbs)
    {
        u_next = pair;
        r = min(pair * w.share, w.n_rest * kbs);
        r_end = min(r + w.share, w.n_rest * kbs);
        part = -1;
    }
    __device__ __forceinline__ bool next(const WideArgs &w, int pairs, int kbs)
    {
        if (u_next < w.n_whole) {
            u = u_next;
            u_next += pairs;
            kb0 = 0;
            kb1 = kbs;
            return true;
        }
        if (r >= r_end) return false;
        const int t = r / kbs;
        u = w.n_whole + t;
        kb0 = r - t * kbs;
        kb1 = min(kbs, kb0 + r_end - r);
        r += kb1 - kb0;
        ++part;
        return true;
    }
    __device__ __forceinline__ uint32_t blocks(const WideArgs &w, int pair, int pairs, int kbs) const   // of all pieces
    {
        return (uint32_t)(pair < w.n_whole ? (w.n_whole - pair + pairs - 1) / pairs : 0) * (uint32_t)kbs + (uint32_t)(r_end - r);
    }
};

// this thread's loads so far have arrived, in `r` (which the compiler may not use before)
__device__ __forceinline__ void tmem_wait16(uint32_t (&r)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :
                 : "memory");
}

// acc += r * f, or r * f * sbs[column] (16 columns)
template <bool PER_ROW>
__device__ __forceinline__ void join16(float2 *acc, const uint32_t (&r)[16], float f, const float *sbs)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float2 f0 = make_float2(f, f), f1 = f0;
        if (PER_ROW) {
            const float4 s4 = reinterpret_cast<const float4 *>(sbs)[j];
            f0 = __fmul2_rn(f0, make_float2(s4.x, s4.y));
            f1 = __fmul2_rn(f1, make_float2(s4.z, s4.w));
        }
        const uint32_t *p = r + j * 4;
        acc[j * 2] = __ffma2_rn(make_float2(__uint_as_float(p[0]), __uint_as_float(p[1])), f0, acc[j * 2]);
        acc[j * 2 + 1] = __ffma2_rn(make_float2(__uint_as_float(p[2]), __uint_as_float(p[3])), f1, acc[j * 2 + 1]);
    }
}

// 4 bytes of global memory into shared memory, asynchronously; zero where !valid
__device__ __forceinline__ void copy4(float *dst, const float *src, bool valid)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(saddr(dst)), "l"(src), "r"(valid ? 4 : 0) : "memory");
}

// 32 rows x 128 bytes of a finished tile from this warp's staging buffer to a result whose rows no bulk copy can take
template <typename T>
__device__ __forceinline__ void store_rows(const unsigned char *stage, T *out, int64_t ldc, int m, int M, int n, int N)
{
    // (four rows of reads before their writes: 3091 x 25533 x 1739, bf16, 190 us, one row at a time 254; N = 25536: 162 us)
    constexpr int E = 16 / sizeof(T), W = 128 / sizeof(T), Q = W / 32, R = 4;     // elements per 16 bytes, per row; of a lane
    const int lane = threadIdx.x & 31;
    T *to = out + (int64_t)m * ldc + n + lane;
#pragma unroll 1
    for (int r0 = 0; r0 < 32; r0 += R) {
        T v[R][Q];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const int e = q * 32 + lane;
                v[r][q] = *reinterpret_cast<const T *>(stage + (r0 + r) * 128 + (((e / E) ^ ((r0 + r) & 7)) << 4) + (e % E) * sizeof(T));
            }
#pragma unroll
        for (int r = 0; r < R; ++r, to += ldc)
#pragma unroll
            for (int q = 0; q < Q; ++q)
                if (m + r0 + r < M && n + q * 32 + lane < N) to[q * 32] = v[r][q];
    }
}

template <bool PER_ROW>
__global__ void __launch_bounds__(kWideThreads, 1)
wide_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
            const __grid_constant__ CUtensorMap map_c, const WideArgs w)
{
    const Args &a = w.a;
    constexpr int kGroup = Scales<PER_ROW>::kGroup, kFloats = Scales<PER_ROW>::kFloats, kGroupFloats = kGroup * kFloats;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ WideSmem sm;
    unsigned char *ring = smem_raw + ((1024u - (saddr(smem_raw) & 1023u)) & 1023u);
    float *scales = reinterpret_cast<float *>(ring + kWideStages * kWideStage + kEpiWarps * kStageOut);   // [2][kGroup][kFloats]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kWideStages; ++s) {
            barrier_init(&sm.full[s], 1);
            barrier_init(&sm.empty[s], 2);                      // both halves' products
        }
        for (int b = 0; b < 2; ++b) {
            for (int g = 0; g < 2; ++g) {
                barrier_init(&sm.tmem_full[g][b], 1);
                barrier_init(&sm.pair_empty[g][b], kEpiWarps);  // half of each block's warps
            }
            barrier_init(&sm.scale_full[b], 1);
            barrier_init(&sm.scale_empty[b], kEpiWarps);
            barrier_init(&sm.nobody[b], 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) tmem_alloc_all_pair(&sm.tmem_base);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_barrier();                                          // the other block's barriers are ready too
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = sm.tmem_base;
    const int kbs = a.kb_total;
    const int rank = (int)cluster_rank(), pair = blockIdx.x / 2, pairs = gridDim.x / 2;
    Piece piece;
    piece.init(w, pair, kbs);
    grid_dependents_may_launch();                               // join_kernel, which waits for the end of this one

    // registers of the first eight warps go to the epilogue: 256 x 32 + 512 x 104 = 768 x 80
    if (warp < 8) asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
    if (warp == 0) {
        if (lane == 0) {
            bool alive = true;
            uint32_t it = 0, s = 0, parity = 1;                 // (waiting for the phase before the first returns at once)
            while (alive && piece.next(w, pairs, kbs)) {
                const int2 t = tile_of(piece.u, a.m_tiles, a.n_tiles, w.gm, w.gn);
                for (int kb = piece.kb0; kb < piece.kb1; ++kb, ++it) {
                    wait_alive(alive, &sm.empty[s], parity, a.status);
                    if (!alive) break;
                    unsigned char *stage = ring + (size_t)s * kWideStage;
                    // (bytes of the other block may be counted before they are announced: the phase cannot end
                    // without the leader's arrival)
                    if (rank == 0) barrier_expect_tx(&sm.full[s], 2u * kWideStage);
                    const uint32_t bar = leader_addr(&sm.full[s]);
                    tma_load_2d_pair(stage, &map_a, kb * kBlockK, t.x * kPairM + rank * kBM, bar);
                    // of the 128 columns of each half, 64 rows of B come from either block
                    tma_load_2d_pair(stage + kWideA, &map_b, kb * kBlockK, t.y * kBN + rank * 64, bar);
                    tma_load_2d_pair(stage + kWideA + kWideB / 2, &map_b, kb * kBlockK, t.y * kBN + 128 + rank * 64, bar);
                    if (++s == kWideStages) { s = 0; parity ^= 1; }
                }
            }
            // copies in flight land before the block may end
            if (rank == 0)
                for (uint32_t i = it > kWideStages ? it - kWideStages : 0; i < it; ++i)
                    wait(&sm.full[i % kWideStages], (i / kWideStages) & 1, a.status);
            // and so do the last arrivals on this block's barriers, which no load waited for
            for (uint32_t i = it > kWideStages ? it - kWideStages : 0; i < it; ++i)
                wait_alive(alive, &sm.empty[i % kWideStages], (i / kWideStages) & 1, a.status);
        }
        __syncwarp();
    } else if (warp >= 4 && warp < 8) {
        // One issuer per accumulator: while one waits, the others' products run. No order is needed between them.
        if (rank == 0) {
            constexpr uint32_t idesc = instr_desc_e4m3(kPairM, kBN / 2);
            const uint32_t g = warp & 1, buf = (warp >> 1) & 1;
            const uint64_t desc0 = smem_desc(saddr(ring), 16, 1024);
            const uint32_t total = piece.blocks(w, pair, pairs, kbs);
            const uint32_t tmem_d = tmem_base + buf * kBN + g * (kBN / 2);
            bool alive = true;
            uint32_t s = buf, s_parity = 0, b_parity = 1;
            for (uint32_t it = buf; it < total && !withheld(kProducts, it, 2); it += 2) {
                wait_alive(alive, &sm.full[s], s_parity, a.status);
                wait_alive(alive, &sm.pair_empty[g][buf], b_parity, a.status);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                // rows 64 g .. of either block's 128 rows of B
                const uint64_t ad = desc0 + s * (kWideStage >> 4), bd = ad + ((kWideA + g * (kWideB / 2)) >> 4);
                if (elect_one() && alive) {                     // (the same lane every time)
#pragma unroll
                    for (int kk = 0; kk < kBlockK / 32; ++kk) mma_f8_pair(tmem_d, ad + kk * 2, bd + kk * 2, idesc, kk ? 1u : 0u);
                    commit_pair(&sm.tmem_full[g][buf]);
                    commit_pair(&sm.empty[s]);
                }
                __syncwarp();
                s += 2;
                if (s >= kWideStages) { s -= kWideStages; s_parity ^= 1; }
                b_parity ^= (uint32_t)alive;
            }
            // every product has ended before tensor memory is freed (b_parity is now that of the last one's phase, or that of the
            // phase before the first)
            if (elect_one()) wait(&sm.tmem_full[g][buf], b_parity, a.status);
        }
        __syncwarp();
    } else if (warp == 1) {
        bool alive = true;
        uint32_t g = 0, parity = 1;
        while (alive && piece.next(w, pairs, kbs)) {
            const int2 t = tile_of(piece.u, a.m_tiles, a.n_tiles, w.gm, w.gn);
            const int m0 = t.x * kPairM + rank * kBM, n0 = t.y * kBN;
            for (int kb0 = piece.kb0; kb0 < piece.kb1; kb0 += kGroup) {
                wait_alive(alive, &sm.scale_empty[g], parity, a.status);
                alive = __all_sync(0xffffffffu, alive);
                if (!alive) break;
                float *to = scales + g * kGroupFloats;
                for (int kb = kb0; kb < min(kb0 + kGroup, piece.kb1); ++kb, to += kFloats) {
                    const float *pa = a.sa + (int64_t)kb * a.M;
#pragma unroll
                    for (int j = lane; j < kBM; j += 32) copy4(to + j, m0 + j < a.M ? pa + m0 + j : a.sa, m0 + j < a.M);
                    if (PER_ROW) {
                        const float *pb = a.sb + (int64_t)kb * a.N;
#pragma unroll
                        for (int j = lane; j < kBN; j += 32) copy4(to + kBM + j, n0 + j < a.N ? pb + n0 + j : a.sb, n0 + j < a.N);
                    } else if (lane < 2) {
                        const int blk = n0 / 128 + lane;
                        const bool in = blk * 128 < a.N;
                        copy4(to + kBM + lane, in ? a.sb + (int64_t)blk * kbs + kb : a.sb, in);
                    }
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
                __syncwarp();
                if (lane == 0 && !withheld(kScaleGroups, (int)g, 1)) barrier_arrive(&sm.scale_full[g]);
                parity ^= g;
                g ^= 1;
            }
        }
    } else if (warp >= 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        const int q = warp & 3, c64 = (warp - 8) >> 2, h = c64 >> 1;   // lanes 32 q .., columns 64 c64 .., their half
        unsigned char *stage = ring + (size_t)kWideStages * kWideStage + (warp - 8) * kStageOut;
        const uint32_t taddr = tmem_base + c64 * 64 + ((uint32_t)(q * 32) << 16);
        bool alive = true, ready = false;                       // ready: the next accumulator is known to be there
        // what this warp's arrivals count on: once it has given up, barriers that nobody waits for (27136 x 50304 x 4096: 0.5 to
        // 1 % for it; arrivals under a condition 2 to 3 %)
        uint32_t pair_empty = leader_addr(&sm.pair_empty[h][0]), scale_empty = saddr(&sm.scale_empty[0]);
        const auto wait_or_leave = [&](unsigned long long *bar, uint32_t parity) {
            if (alive && !wait(bar, parity, a.status)) {
                alive = false;
                pair_empty = leader_addr(&sm.nobody[0]);
                scale_empty = saddr(&sm.nobody[0]);
            }
        };
        uint32_t buf = 0, parity = 0, g = 0, g_parity = 0;
        while (piece.next(w, pairs, kbs)) {
            float2 acc[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) acc[j] = make_float2(0.f, 0.f);
            const float *slot = scales;
            int left = 0;                                       // blocks of K left in the group of scales
#pragma unroll 1
            for (int kb = piece.kb0; kb < piece.kb1; ++kb) {
                if (left == 0) {
                    wait_or_leave(&sm.scale_full[g], g_parity);
                    slot = scales + g * kGroupFloats;
                    left = min(kGroup, piece.kb1 - kb);
                }
                const float f = PER_ROW ? slot[q * 32 + lane] : slot[q * 32 + lane] * slot[kBM + h];
                const float *sbs = slot + kBM + c64 * 64;       // PER_ROW: this warp's 64 factors
                if (!ready) wait_or_leave(&sm.tmem_full[h][buf], parity);
                __syncwarp();
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                uint32_t r[2][16];
                const uint32_t at = taddr + buf * kBN;
                tmem_ld16(at, r[0]);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    tmem_wait16(r[c & 1]);
                    if (c < 3) {
                        tmem_ld16(at + (c + 1) * 16, r[(c + 1) & 1]);
                    } else {
                        // released before the last multiply-adds: what stands between an accumulator's arrival and its
                        // release is on the way from one matrix instruction to the next
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        __syncwarp();
                        barrier_arrive_cluster_if(pair_empty + buf * 8, lane == 0 && !withheld(kReleases, kb - piece.kb0, 2));
                        parity ^= buf;
                        buf ^= 1;
                        ready = peek(&sm.tmem_full[h][buf], parity);
                    }
                    join16<PER_ROW>(acc + c * 8, r[c & 1], f, sbs + c * 16);
                }
                slot += kFloats;
                if (--left == 0) {
                    __syncwarp();
                    if (lane == 0) barrier_arrive_cluster(scale_empty + g * 8);
                    g_parity ^= g;
                    g ^= 1;
                }
            }
            if (!alive) {
#pragma unroll
                for (int j = 0; j < 32; ++j) acc[j].x = acc[j].y = __uint_as_float(0x7fffffffu);
            }
            const int2 t = tile_of(piece.u, a.m_tiles, a.n_tiles, w.gm, w.gn);
            const int n = t.y * kBN + c64 * 64;
            const int m_warp = t.x * kPairM + rank * kBM + q * 32;
            if (piece.part >= 0) {                              // a part of the tile's sum
                // (four columns of 256 rows follow one another: a warp writes 512 bytes at a time)
                float4 *to = reinterpret_cast<float4 *>(w.scratch + (size_t)(pair * 2 + piece.part) * kTileFloats) +
                             c64 * 16 * kPairM + rank * kBM + q * 32 + lane;
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    to[j * kPairM] = make_float4(acc[j * 2].x, acc[j * 2].y, acc[j * 2 + 1].x, acc[j * 2 + 1].y);
                continue;
            }
            // the tile: 64 bf16 or 32 fp32 columns at a time through shared memory, 16-byte piece c of row r at c ^ (r & 7)
            unsigned char *row = stage + lane * 128;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                if (c == 1 && !a.out_f32) break;
                if (lane == 0) tma_store_wait_read();           // the buffer's last copy has read it
                __syncwarp();
                if (a.out_f32) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        *reinterpret_cast<float4 *>(row + ((j ^ (lane & 7)) << 4)) = make_float4(
                            acc[c * 16 + j * 2].x, acc[c * 16 + j * 2].y, acc[c * 16 + j * 2 + 1].x, acc[c * 16 + j * 2 + 1].y);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        uint32_t v[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const __nv_bfloat162 b2 = __float22bfloat162_rn(acc[j * 4 + e]);
                            v[e] = *reinterpret_cast<const uint32_t *>(&b2);
                        }
                        *reinterpret_cast<uint4 *>(row + ((j ^ (lane & 7)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
                    }
                }
                if (n + c * 32 + (a.out_f32 ? 32 : 64) <= w.bulk_cols) {
                    fence_async_proxy();
                    __syncwarp();
                    if (lane == 0 && m_warp < a.M && n + c * 32 < a.N) tma_store_2d(&map_c, n + c * 32, m_warp, stage);
                } else {
                    __syncwarp();
                    if (a.out_f32) store_rows(stage, reinterpret_cast<float *>(a.out), a.ldc, m_warp, a.M, n + c * 32, a.N);
                    else store_rows(stage, reinterpret_cast<__nv_bfloat16 *>(a.out), a.ldc, m_warp, a.M, n, a.N);
                    __syncwarp();
                }
            }
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

// The tiles that were cut along K: a block adds up 32 rows x 64 columns over the pairs that hold parts of them, in the order
// of K, and turns them in shared memory so that rows leave in runs. Launched as a dependent of the wide kernel.
constexpr int kJoinThreads = 256, kJoinBlocks = (kPairM / 32) * (kBN / 64);
__global__ void __launch_bounds__(kJoinThreads)
join_kernel(const WideArgs w)
{
    __shared__ float4 turn[32][17];
    const Args &a = w.a;
    const int rest = blockIdx.x / kJoinBlocks, part_of = blockIdx.x % kJoinBlocks;
    const int row0 = (part_of % (kPairM / 32)) * 32, j0 = part_of / (kPairM / 32) * 16;
    const int2 t = tile_of(w.n_whole + rest, a.m_tiles, a.n_tiles, w.gm, w.gn);
    const int m0 = t.x * kPairM + row0, n0 = t.y * kBN + j0 * 4;
    const int first = rest * a.kb_total / w.share, last = ((rest + 1) * a.kb_total - 1) / w.share;
    const int lane = threadIdx.x & 31, jj = threadIdx.x >> 5;
    grid_dependency_wait();
    if (m0 >= a.M || n0 >= a.N) return;
    float4 v[2];
    v[0] = v[1] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int c = first; c <= last; ++c) {
        const int part = rest - c * w.share / a.kb_total;       // the pair's first or second tile
        const float4 *from = reinterpret_cast<const float4 *>(w.scratch + (size_t)(c * 2 + part) * kTileFloats) + row0 + lane;
        const float4 x = from[(j0 + jj) * kPairM], y = from[(j0 + jj + 8) * kPairM];
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
        const bool vec = n + 4 <= a.N && (reinterpret_cast<uintptr_t>(a.out) & 15u) == 0 && (a.ldc & 3) == 0;
        if (n < a.N) store4(a, m0 + r, n, turn[r][c4], vec);
    }
}

static int pairs_of_device(int *pairs)
{
    int dev = 0, sms = 148;
    PPO_RETURN_IF_CUDA(cudaGetDevice(&dev));
    PPO_RETURN_IF_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    *pairs = sms / 2;
    return PPO_OK;
}

// Tiles left over by the last full round of the pairs are cut along K when that saves each pair 24 blocks of K or more
// (0.3 to 0.5 us each, against about 8 us for writing and joining the parts: 600 x 2000 x 8192 37 us whole, 27 cut; with 16
// blocks saved 2000 x 2000 x 16384 72 whole, 80 cut).
struct WidePlan {
    int m_tiles, n_tiles, n_whole, n_rest, share;
};

static WidePlan wide_plan(int64_t M, int64_t N, int kbs, int pairs)
{
    WidePlan p;
    p.m_tiles = (int)((M + kPairM - 1) / kPairM);
    p.n_tiles = (int)((N + kBN - 1) / kBN);
    const int64_t units = (int64_t)p.m_tiles * p.n_tiles;
    p.n_whole = (int)units;
    p.n_rest = p.share = 0;
    const int rest = (int)(units % pairs);
    const int64_t share = ((int64_t)rest * kbs + pairs - 1) / pairs;
    if (rest > 0 && kbs - share >= 24 && units < ((int64_t)1 << 30)) {
        p.n_rest = rest;
        p.n_whole = (int)units - rest;
        p.share = (int)share;
    }
    return p;
}

static size_t wide_scratch_bytes(const WidePlan &p, int pairs) { return p.share ? (size_t)pairs * 2 * kTileFloats * 4 : 0; }

static int launch_wide(Args a, const void *A, int64_t lda, const void *B, int64_t ldb, int64_t K, float *scratch, cudaStream_t s)
{
    CUtensorMap ma, mb;
    int rc = make_map_8bit(&ma, A, (uint64_t)K, (uint64_t)a.M, (uint64_t)lda, kBM);
    if (rc) return rc;
    rc = make_map_8bit(&mb, B, (uint64_t)K, (uint64_t)a.N, (uint64_t)ldb, 64);
    if (rc) return rc;
    int pairs = 0;
    rc = pairs_of_device(&pairs);
    if (rc) return rc;
    WidePlan p = wide_plan(a.M, a.N, a.kb_total, pairs);
    if (!scratch) {                                             // whole tiles only
        p.n_whole += p.n_rest;
        p.n_rest = p.share = 0;
    }
    const int64_t units = (int64_t)p.m_tiles * p.n_tiles;
    if (units >= ((int64_t)1 << 30)) return PPO_ERR_SHAPE;
    a.m_tiles = p.m_tiles;
    a.n_tiles = p.n_tiles;
    WideArgs w = {};
    w.a = a;
    w.gm = 5;
    w.gn = 16;
    w.n_whole = p.n_whole;
    w.n_rest = p.n_rest;
    w.share = p.share;
    w.scratch = scratch;
    const int64_t pitch = a.ldc * (a.out_f32 ? 4 : 2);
    if (reinterpret_cast<uintptr_t>(a.out) % 16 == 0 && pitch % 16 == 0 && pitch < ((int64_t)1 << 40))
        w.bulk_cols = a.N % (a.out_f32 ? 4 : 8) ? a.N : 0x7fffffff;
    CUtensorMap mc = {};
    if (w.bulk_cols) {
        rc = make_map_out(&mc, a.out, a.out_f32 != 0, (uint64_t)a.N, (uint64_t)a.M, (uint64_t)pitch, 32);
        if (rc) return rc;
    }
    auto kern = a.per_row ? wide_kernel<true> : wide_kernel<false>;
    PPO_RETURN_IF_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kWideSmem));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * (p.share || units > pairs ? pairs : (int)units)));
    cfg.blockDim = dim3(kWideThreads);
    cfg.dynamicSmemBytes = kWideSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    PPO_RETURN_IF_CUDA(cudaLaunchKernelEx(&cfg, kern, ma, mb, mc, w));
    if (!p.share) return PPO_OK;
    PPO_RETURN_IF_CUDA(launch_dependent(join_kernel, dim3((unsigned)(p.n_rest * kJoinBlocks)), dim3(kJoinThreads), 0, s, w));
    return PPO_OK;
}

// Rows of A in a tile of the narrow kernel, or 0 for the wide one. The wide kernel takes its time per block of K and tile
// whatever the SMs without a tile do; while there are so few 128 x 64 tiles that two blocks or more can share the K of
// each, those are faster (64 x 4096 x 8192: 13 against 38 us, 200 x 4096 x 8192: 27 against 39; with a block for each:
// 400 x 4096 x 8192 55 against 39).
static int narrow_rows(int64_t M, int64_t N)
{
    if (M <= 32) return M <= 16 ? 16 : 32;
    return ((M + 63) / 64) * ((N + 127) / 128) * 2 <= narrow_places<64>() ? 64 : 0;
}

}   // namespace fp8
}   // namespace ppo

using namespace ppo;

extern "C" size_t ppo_fp8_scratch_bytes(int64_t M, int64_t N, int64_t K)
{
    const int64_t limit = ((int64_t)1 << 31) - 512;
    if (M <= 0 || N <= 0 || K <= 0 || M >= limit || N >= limit || K >= limit || fp8::narrow_rows(M, N)) return 0;
    int pairs = 0;
    if (fp8::pairs_of_device(&pairs) != PPO_OK) {
        (void)cudaGetLastError();
        pairs = 74;
    }
    return fp8::wide_scratch_bytes(fp8::wide_plan(M, N, (int)((K + 127) / 128), pairs), pairs);
}

extern "C" int ppo_fp8_matmul(const void *A, int64_t lda, const float *a_scales, const void *B, int64_t ldb,
                              const float *b_scales, int block_n, int64_t M, int64_t N, int64_t K, void *C,
                              int out_dtype, int64_t ldc, void *workspace, void *scratch, void *stream)
{
    if (out_dtype != PPO_F32 && out_dtype != PPO_BF16) return PPO_ERR_DTYPE;
    const int64_t limit = ((int64_t)1 << 31) - 512;
    if (M < 0 || N <= 0 || K <= 0 || M >= limit || N >= limit || K >= limit || lda < K || ldb < K || ldc < N ||
        lda % 16 || ldb % 16)
        return PPO_ERR_SHAPE;
    if (block_n != 1 && block_n != 128) return PPO_ERR_PARAM;
    if (M == 0) return PPO_OK;
    if (!A || !a_scales || !B || !b_scales || !C) return PPO_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(A) % 16 || reinterpret_cast<uintptr_t>(B) % 16 ||
        reinterpret_cast<uintptr_t>(C) % (out_dtype == PPO_F32 ? 4 : 2) || reinterpret_cast<uintptr_t>(scratch) % 256)
        return PPO_ERR_ALIGN;
    fp8::Args a = {};
    a.M = (int)M;
    a.N = (int)N;
    a.kb_total = (int)((K + 127) / 128);
    a.sa = a_scales;
    a.sb = b_scales;
    a.per_row = block_n == 1;
    a.out = C;
    a.ldc = ldc;
    a.out_f32 = out_dtype == PPO_F32;
    a.status = workspace ? &ws_header(workspace)->status : nullptr;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    switch (fp8::narrow_rows(M, N)) {
    case 16: return fp8::launch_narrow<16>(a, A, lda, B, ldb, K, s);
    case 32: return fp8::launch_narrow<32>(a, A, lda, B, ldb, K, s);
    case 64: return fp8::launch_narrow<64>(a, A, lda, B, ldb, K, s);
    }
    return fp8::launch_wide(a, A, lda, B, ldb, K, reinterpret_cast<float *>(scratch), s);
}
