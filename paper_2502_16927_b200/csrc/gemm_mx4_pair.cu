// Product of two microscaled 4-bit matrices on CTA pairs (tcgen05 cta_group::2), for large dense ones: C = sigma(A W^T), fp32 sums.
//
// Two CTAs of a cluster own a 256 x 256 tile of C: each has 128 rows of A and 128 rows of W in its shared memory, and the 128 x 256
// accumulator of its rows.  What bounds the one-CTA kernel is shared memory: a 128 x 128 tile reads 8 KB of codes for 64 cycles of the tensor pipe
// (64 columns) and takes as many in, twice what shared memory gives; here the same 8 KB serve 128 cycles.  Every CTA holds the scale bytes of
// its own rows of A and of all 256 rows of W (its half of the products needs them all); the leader's copies to tensor memory (cta_group::2) move
// both CTAs'.  An accumulator of 256 columns and the scale bytes leave no room for a second one: all sixteen epilogue warps empty it into registers
// at once, and what they do with it runs beside the next tile's products.  Barriers as in gemm_tc2.cu: loads of both CTAs complete on the
// leader's, commits arrive at both.  No TMA multicast.
#include "gemm_mx4.cuh"

namespace bigmac {

using namespace mx4;

namespace {

constexpr int kBN = 256, kStages = 4, kSliceBytes = 128 * 128;           // a CTA's rows of A, and of W, in a slice of 256 columns
constexpr int kEpiPair = 16;
constexpr int kThreadsPair = (2 + kEpiPair) * 32;
constexpr uint32_t kSfBytes = 2 * kSfTile * 3;                           // A's row tile, W's two; two k tiles each
constexpr uint32_t kStageBytes = 2 * kSliceBytes + kSfBytes;
constexpr uint32_t kBoxPair = 32 * 64 * 2;
constexpr uint32_t kSfColPair = kBN, kTmemPair = 512;                    // scale bytes behind the accumulator: A's 8 columns, W's 16
constexpr size_t kSmemPair = 1024 + kStages * kStageBytes + kEpiPair * kBoxPair + (2 * kStages + 2) * 8 + 16;
static_assert(kStageBytes % 1024 == 0 && kSmemPair <= 227 * 1024, "shared memory of a block");

__device__ __forceinline__ void copy_scales_pair(uint32_t tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void umma_mx4_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
}
// As instr_desc_mx4, M 256.
__host__ __device__ constexpr uint32_t instr_desc_mx4_pair(int half) {
    return ((uint32_t)(2 * half) << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kBN >> 3) << 17) | (1u << 23) | ((uint32_t)(256 >> 4) << 24) |
           ((uint32_t)(2 * half) << 29);
}

template <int OUT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreadsPair, 1)
gemm_mx4_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_sa,
                     const __grid_constant__ CUtensorMap map_sw, const __grid_constant__ CUtensorMap map_c, const Mx4Params p) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* boxes_c = smem + kStages * kStageBytes;
    uint64_t* full_bar = (uint64_t*)(boxes_c + kEpiPair * kBoxPair);     // waited on in the leader only
    uint64_t* empty_bar = full_bar + kStages;
    uint64_t* tmem_full_bar = empty_bar + kStages;
    uint64_t* tmem_empty_bar = tmem_full_bar + 1;                        // the leader's is used
    uint32_t* tmem_slot = (uint32_t*)(tmem_empty_bar + 1);
    volatile int* dead = (volatile int*)(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;
    if (threadIdx.x == 32) {
        prefetch_tensormap(&map_a);
        prefetch_tensormap(&map_w);
        prefetch_tensormap(&map_sa);
        prefetch_tensormap(&map_sw);
        prefetch_tensormap(&map_c);
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { mbar_init(&full_bar[s], 1); mbar_init(&empty_bar[s], 1); }
        mbar_init(tmem_full_bar, 1);
        mbar_init(tmem_empty_bar, 2 * kEpiPair);
        *dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) tmem_alloc_pair(tmem_slot, kTmemPair);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                                                  // the peer's barriers exist before anything signals them
    grid_dependency_launch();
    grid_dependency_wait();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const int ktiles = mx4_ktiles(p.K), num_kb = (p.K + kSliceK - 1) / kSliceK;
    const int tiles_n = (p.N + kBN - 1) / kBN, total = (p.M + 255) / 256 * tiles_n;
    const int first = blockIdx.x >> 1, step = gridDim.x >> 1;

    if (warp == 0) {
        // ------------------------------------------------------------------ producer (both CTAs)
        if (elect_one()) {
            uint32_t s = 0, phase = 1;
            for (int t = first; t < total; t += step) {
                const int mt = 2 * (t / tiles_n) + (int)rank, n0 = t % tiles_n * kBN;
                for (int kb = 0; kb < num_kb; ++kb, s = (s + 1 == kStages ? 0 : s + 1), phase ^= (s == 0)) {
                    mbar_wait_lean(&empty_bar[s], phase, dead, p.status);
                    if (leader) mbar_expect_tx(&full_bar[s], 2 * kStageBytes);
                    const uint32_t bar = map_to_cta(&full_bar[s], 0);
                    uint8_t* a = smem + s * kStageBytes;
                    uint8_t* f = a + 2 * kSliceBytes;
                    tma_load_2d_pair(a, &map_a, bar, kb * 128, mt * 128);
                    tma_load_2d_pair(a + kSliceBytes, &map_w, bar, kb * 128, n0 + (int)rank * 128);
                    tma_load_2d_pair(f, &map_sa, bar, 0, mt * ktiles + 2 * kb);
                    tma_load_2d_pair(f + 2 * kSfTile, &map_sw, bar, 0, n0 / 128 * ktiles + 2 * kb);
                    tma_load_2d_pair(f + 4 * kSfTile, &map_sw, bar, 0, (n0 / 128 + 1) * ktiles + 2 * kb);
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ scale bytes and products (one thread of the leader)
        if (leader && elect_one()) {
            const uint64_t da0 = smem_desc(smem_u32(smem), 16, 1024), db0 = smem_desc(smem_u32(smem + kSliceBytes), 16, 1024);
            const uint64_t df0 = scale_desc(smem_u32(smem + 2 * kSliceBytes));
            const uint32_t fa = tmem + kSfColPair, fw = fa + 8;
            uint32_t stage = 0, phase = 0, use = 0;
            for (int t = first; t < total; t += step, ++use) {
                for (int kb = 0; kb < num_kb; ++kb) {
                    mbar_wait_lean(&full_bar[stage], phase, dead, p.status);
                    tc_fence_after();
                    const uint64_t at = (uint64_t)stage * (kStageBytes >> 4);
                    const int cols = min(kSliceK, p.K - kb * kSliceK);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if (j * 128 >= cols) break;
                        copy_scales_pair(fa + 4 * j, df0 + at + j * (kSfTile >> 4));
#pragma unroll
                        for (int i = 0; i < 2; ++i) copy_scales_pair(fw + 4 * (2 * j + i), df0 + at + ((2 * (1 + i) + j) * (kSfTile >> 4)));
                    }
                    if (kb == 0) {                                       // the accumulator is free only now: the first slice did not wait for it
                        mbar_wait_cluster(tmem_empty_bar, (use & 1) ^ 1, dead, p.status);
                        tc_fence_after();
                    }
#pragma unroll
                    for (int kk = 0; kk < kSliceK / 64; ++kk) {
                        if (kk * 64 >= cols) break;
                        umma_mx4_pair(tmem, da0 + at + kk * 2, db0 + at + kk * 2, instr_desc_mx4_pair(kk & 1), fa + 4 * (kk >> 1), fw + 8 * (kk >> 1),
                                      kb != 0 || kk != 0);
                    }
                    umma_commit_pair(&empty_bar[stage]);
                    if (++stage == kStages) { stage = 0; phase ^= 1; }
                }
                umma_commit_pair(tmem_full_bar);
            }
        }
    } else {
        // ------------------------------------------------------------------ epilogue (both CTAs): 32 rows and 64 columns a warp
        const int quad = warp & 3, part = (warp - 2) >> 2;
        Mx4Epilogue<OUT, 64> epi(p, &map_c, boxes_c + (warp - 2) * kBoxPair, lane);
        const uint32_t t_addr = tmem + ((uint32_t)(quad * 32) << 16) + part * 64, leader_empty = map_to_cta(tmem_empty_bar, 0);
        uint32_t use = 0;
        for (int t = first; t < total; t += step, ++use) {
            const int row0 = (2 * (t / tiles_n) + (int)rank) * 128 + quad * 32, col0 = t % tiles_n * kBN + part * 64;
            mbar_wait_lean(tmem_full_bar, use & 1, dead, p.status);
            tc_fence_after();
            float v[2][32];
            tmem_load_32_nowait(t_addr, (uint32_t*)v[0]);
            tmem_load_32_nowait(t_addr + 32, (uint32_t*)v[1]);
            tmem_load_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(leader_empty);
            epi.begin(col0, row0, p.M - row0, row0);
            epi.chunk(0, v[0]);
            epi.chunk(1, v[1]);
            epi.end();
        }
        epi.finish();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                                                  // both CTAs are done with the pair's tensor memory and barriers
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem, kTmemPair);
    }
}

// Scale bytes as rows of 128 words, a tile each; two tiles a box.
bool make_map_scales(CUtensorMap* map, const void* base, uint64_t tiles) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {128, tiles}, strides[1] = {kSfTile};
    const cuuint32_t box[2] = {128, 2}, elem[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<void*>(base), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int OUT>
cudaError_t launch_pair(const Mx4View& a, const Mx4View& w, Mx4Params p, cudaStream_t stream) {
    CUtensorMap ma, mw, msa, msw, mc;
    const uint64_t row = (uint64_t)p.K / 2, ktiles = mx4_ktiles(p.K);
    if (!make_map_u8(&ma, a.codes, row, p.M, row, 128, 128, CU_TENSOR_MAP_SWIZZLE_128B) || !make_map_u8(&mw, w.codes, row, p.N, row, 128, 128, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_map_scales(&msa, a.scales, (uint64_t)(p.M + 127) / 128 * ktiles) || !make_map_scales(&msw, w.scales, (uint64_t)(p.N + 127) / 128 * ktiles))
        return cudaErrorInvalidValue;
    p.tma_store = OUT <= OUT_BF16_ACT && tma_store_ok(p);
    mc = mw;
    if (p.tma_store && !make_map(&mc, p.C, (uint64_t)p.N, (uint64_t)p.M, (uint64_t)p.ldc, 64, 32, CU_TENSOR_MAP_SWIZZLE_128B)) return cudaErrorInvalidValue;
    static PerDeviceOnce once;
    auto kernel = gemm_mx4_pair_kernel<OUT>;
    int dev;
    if (once.needed(&dev)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemPair);
        if (e != cudaSuccess) return e;
        once.mark(dev);
    }
    const int64_t total = (int64_t)((p.M + 255) / 256) * ((p.N + kBN - 1) / kBN), pairs = gemm_tc_sm_count() / 2;
    return launch_chained(kernel, 2 * (int)(total < pairs ? total : pairs), kThreadsPair, kSmemPair, stream, ma, mw, msa, msw, mc, p);
}

}  // namespace

cudaError_t launch_mx4_matmul_pair(const Mx4View& a, const Mx4View& w, const Mx4Params& p, int dtype, cudaStream_t stream) {
    if (p.out_codes) return p.act == BIGMAC_ACT_GELU_ERF ? launch_pair<OUT_MX4_GELU>(a, w, p, stream) : launch_pair<OUT_MX4>(a, w, p, stream);
    if (dtype == BIGMAC_F32) return launch_pair<OUT_F32>(a, w, p, stream);
    if (p.act == BIGMAC_ACT_IDENTITY) return launch_pair<OUT_BF16>(a, w, p, stream);
    return p.act == BIGMAC_ACT_GELU_ERF ? launch_pair<OUT_BF16_GELU>(a, w, p, stream) : launch_pair<OUT_BF16_ACT>(a, w, p, stream);
}

}  // namespace bigmac
