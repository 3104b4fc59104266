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

// A wait that is skipped once one has run out: the block then reaches its end quickly, with the same control flow.
__device__ __forceinline__ void wait_alive(bool &alive, unsigned long long *bar, uint32_t parity, int *status)
{
    if (alive) alive = wait(bar, parity, status);
}

constexpr int kNarrowStages = 6, kNarrowBufs = 2, kNarrowThreads = 192;

template <int MT>
struct NarrowSmem {
    unsigned long long full[kNarrowStages], empty[kNarrowStages], tmem_full[kNarrowBufs], tmem_empty[kNarrowBufs];
    uint32_t tmem_base;
    float4 scale[4][kNarrowBufs][MT / 4];     // per epilogue warp: the columns' factors of a block of K
};

template <int MT> __host__ __device__ constexpr int narrow_stage_bytes() { return (128 + MT) * kBlockK; }
// accumulator columns: a power of two, at least 32
template <int MT> __host__ __device__ constexpr uint32_t narrow_columns() { return kNarrowBufs * MT < 32 ? 32 : kNarrowBufs * MT; }

template <int MT>
__global__ void __launch_bounds__(kNarrowThreads)
narrow_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const Args a, int split)
{
    constexpr int kStage = narrow_stage_bytes<MT>();
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ NarrowSmem<MT> sm;
    unsigned char *ring = smem_raw + ((1024u - (saddr(smem_raw) & 1023u)) & 1023u);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = blockIdx.x % split, tile = blockIdx.x / split;
    const int m0 = (tile % a.m_tiles) * MT, n0 = (tile / a.m_tiles) * 128;
    const int kb0 = (int)((int64_t)a.kb_total * rank / split), kb1 = (int)((int64_t)a.kb_total * (rank + 1) / split);

    if (threadIdx.x == 0) {
        for (int s = 0; s < kNarrowStages; ++s) {
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
                const int s = issued % kNarrowStages;
                if (issued >= kNarrowStages) wait_alive(alive, &sm.empty[s], ((issued / kNarrowStages) - 1) & 1, a.status);
                if (!alive) break;
                unsigned char *stage = ring + (size_t)s * kStage;
                barrier_expect_tx(&sm.full[s], (uint32_t)kStage);
                tma_load_2d(stage, &map_b, kb * kBlockK, n0, &sm.full[s]);
                tma_load_2d(stage + 128 * kBlockK, &map_a, kb * kBlockK, m0, &sm.full[s]);
            }
            // copies in flight land before the block may end
            for (int i = issued > kNarrowStages ? issued - kNarrowStages : 0; i < issued; ++i)
                wait(&sm.full[i % kNarrowStages], (i / kNarrowStages) & 1, a.status);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr uint32_t idesc = instr_desc_e4m3(128, MT);
            bool alive = true;
            for (int i = 0; i < kb1 - kb0; ++i) {
                const int s = i % kNarrowStages, buf = i % kNarrowBufs;
                if (i >= kNarrowBufs) wait_alive(alive, &sm.tmem_empty[buf], ((i / kNarrowBufs) - 1) & 1, a.status);
                wait_alive(alive, &sm.full[s], (i / kNarrowStages) & 1, a.status);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t b_addr = saddr(ring + (size_t)s * kStage), a_addr = b_addr + 128 * kBlockK;
#pragma unroll
                for (int kk = 0; kk < kBlockK / 32; ++kk)
                    mma_f8(tmem_base + buf * MT, smem_desc(b_addr + kk * 32, 16, 1024), smem_desc(a_addr + kk * 32, 16, 1024),
                           idesc, kk ? 1u : 0u);
                commit(&sm.empty[s]);
                commit(&sm.tmem_full[buf]);
            }
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
                    if (lane == 0) barrier_arrive(&sm.tmem_empty[buf]);
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
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        tmem_free(tmem_base, narrow_columns<MT>());
    }
    // every copy has landed and every product is done: the ring is free for the join
    const int q = warp & 3, nl = q * 32 + lane, n = n0 + nl;
    if (split > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        float *part = reinterpret_cast<float *>(ring);             // [MT][128]
        if (warp >= 2) {
#pragma unroll
            for (int j = 0; j < MT; ++j) part[j * 128 + nl] = acc[j];
        }
        cluster.sync();
        if (warp >= 2) {
            for (int j = rank; j < MT; j += split) {
                float v = 0.f;
                for (int r = 0; r < split; ++r) v += cluster.map_shared_rank(part, r)[j * 128 + nl];
                const int m = m0 + j;
                if (m < a.M && n < a.N) {
                    if (a.out_f32) reinterpret_cast<float *>(a.out)[(int64_t)m * a.ldc + n] = v;
                    else reinterpret_cast<__nv_bfloat16 *>(a.out)[(int64_t)m * a.ldc + n] = __float2bfloat16_rn(v);
                }
            }
        }
        cluster.sync();
    } else if (warp >= 2 && n < a.N) {
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
    int split = 1;
    while (split < 8 && tiles * split < 2 * 148 && a.kb_total >= 4 * split) split *= 2;
    if (tiles * split >= ((int64_t)1 << 31)) return PPO_ERR_SHAPE;
    const size_t smem = (size_t)kNarrowStages * narrow_stage_bytes<MT>() + 1024;
    PPO_RETURN_IF_CUDA(cudaFuncSetAttribute(narrow_kernel<MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * split));
    cfg.blockDim = dim3(kNarrowThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = split > 1 ? 1 : 0;
    PPO_RETURN_IF_CUDA(cudaLaunchKernelEx(&cfg, narrow_kernel<MT>, ma, mb, a, split));
    return PPO_OK;
}

}   // namespace fp8
}   // namespace ppo

using namespace ppo;

extern "C" int ppo_fp8_matmul(const void *A, int64_t lda, const float *a_scales, const void *B, int64_t ldb,
                              const float *b_scales, int block_n, int64_t M, int64_t N, int64_t K, void *C,
                              int out_dtype, int64_t ldc, void *workspace, void *stream)
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
        reinterpret_cast<uintptr_t>(C) % (out_dtype == PPO_F32 ? 4 : 2))
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
    if (M <= 16) return fp8::launch_narrow<16>(a, A, lda, B, ldb, K, s);
    return fp8::launch_narrow<64>(a, A, lda, B, ldb, K, s);
}
