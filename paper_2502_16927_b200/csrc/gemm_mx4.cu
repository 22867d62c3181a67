// Product of two microscaled 4-bit matrices on the tensor cores (layout: mx4.h):
//
//   C[m, n] = sigma( sum_k A(m, k) W(n, k) ),   A(m, k) = e2m1 code * 2^(s - 127) of its block of 32, W alike
//
// tcgen05.mma kind::mxf4 takes both operands as codes (64 columns an instruction) and multiplies the blocks' scales in; sums are fp32 in
// tensor memory.  Dense, or grouped: A holds the segments of E experts, W their E matrices, and C the rows in the caller's order.
//
// Persistent CTAs walk the 128 x BN tiles of C.  Warp 0 streams slices of 256 columns into a ring of stages: codes by TMA (128 bytes a
// row, 128-byte swizzle), scale bytes by bulk copies (512 bytes for 128 rows and 128 columns).  Warp 1 moves a slice's scale
// bytes to tensor memory (tcgen05.cp, in order before the products that read them, as the products before it are in order before the
// copy: one buffer is enough) and issues the products.  Two sets of eight warps drain the two accumulators in turn, each while the other's
// fills and the other set stores: with all sixteen on one accumulator every latency of a tile (barrier, tensor memory, stores) was waited out
// by all (131072 rows, r 256 -> h 1024: 142 us).  bf16 rows leave through shared memory and TMA, 128 bytes a row; 32-byte stores of the
// lanes' own rows alone took 1350 cycles a tile.
#include "gemm_mx4.cuh"

namespace bigmac {

using namespace mx4;

namespace {

template <int BN, int STAGES>
struct Mx4Smem {
    static constexpr uint32_t kBBytes = BN * 128;
    static constexpr uint32_t kSfBytes = 2 * kSfTile * 2;                // two k tiles of A's row tile, then of W's
    static constexpr uint32_t kStage = kABytes + kBBytes + kSfBytes;     // a multiple of 1024
    static_assert(kStage % 1024 == 0, "128-byte swizzle: stages on 1024-byte boundaries");
    static constexpr int kCols = BN / 2;                                 // columns of an epilogue warp
    static constexpr uint32_t kBox = 32 * kCols * 2;
    static constexpr uint32_t kBars = (2 * STAGES + 4) * 8 + 16;
    static constexpr size_t bytes(int E) { return 1024 + STAGES * kStage + kEpi * kBox + kBars + (size_t)(2 * E + 2) * 4; }
};

template <int BN, int STAGES, int OUT>
__global__ void __launch_bounds__(kThreadsMx4, 1)
gemm_mx4_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_w,
                const __grid_constant__ CUtensorMap map_c, const Mx4Params p) {
    using S = Mx4Smem<BN, STAGES>;
    constexpr uint32_t kSfCol = 2 * BN;                                  // scale bytes behind them: A's 8 columns, then W's
    constexpr uint32_t kTmemCols = kSfCol + 16 <= 256 ? 256 : 512;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* boxes_c = smem + STAGES * S::kStage;
    uint64_t* full_bar = (uint64_t*)(boxes_c + kEpi * S::kBox);
    uint64_t* empty_bar = full_bar + STAGES;
    uint64_t* tmem_full_bar = empty_bar + STAGES;                        // [2]
    uint64_t* tmem_empty_bar = tmem_full_bar + 2;                        // [2]
    uint32_t* tmem_slot = (uint32_t*)(tmem_empty_bar + 2);
    volatile int* dead = (volatile int*)(tmem_slot + 1);
    int32_t* tables = (int32_t*)(tmem_slot + 4);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 32) {
        prefetch_tensormap(&map_a);
        prefetch_tensormap(&map_w);
        prefetch_tensormap(&map_c);
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&full_bar[s], 1); mbar_init(&empty_bar[s], 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(&tmem_full_bar[s], 1); mbar_init(&tmem_empty_bar[s], kEpi / 2); }
        *dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(tmem_slot, kTmemCols);
    tc_fence_before();
    __syncthreads();
    grid_dependency_launch();
    grid_dependency_wait();
    Mx4Segments seg{};
    if (p.offsets) seg.load(tables, p.offsets, p.E, p.M);
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const int ktiles = mx4_ktiles(p.K), num_kb = (p.K + kSliceK - 1) / kSliceK;
    const int tiles_n = (p.N + BN - 1) / BN;
    const int tiles_m = p.offsets ? (int)min((int64_t)seg.tiles[p.E], p.capacity / kMx4Tile) : (p.M + kMx4Tile - 1) / kMx4Tile;
    const int total = tiles_m * tiles_n;
    // The CTAs side by side along rows of tiles, which share their codes in L2; grouped with few tiles a CTA: a run of tiles each, so that an expert is
    // looked up once (a step of the grid crosses 18 of 64 experts at 1024 columns: 512 rows 10.8 us, in runs 9.5).  With more, runs spread the CTAs
    // over more weights than L2 holds (65536 rows of 128 experts, h 2048 -> r 512, 16 tiles a CTA: 57 us, in runs 69).
    const bool runs = p.offsets && total <= 4 * (int)gridDim.x;
    const int first = runs ? (int)((int64_t)total * blockIdx.x / gridDim.x) : (int)blockIdx.x, step = runs ? 1 : (int)gridDim.x;
    const int last = runs ? (int)((int64_t)total * (blockIdx.x + 1) / gridDim.x) : total;

    if (warp == 0) {
        // ------------------------------------------------------------------ producer
        if (elect_one()) {
            const int w_row_tiles = (p.N + 127) / 128;
            uint32_t s = 0, phase = 1;
            Mx4Walk walk;
            walk.init(first, step, tiles_n);
            for (int t = first; t < last; t += step, walk.next()) {
                const Mx4Rows q = mx4_rows(p, seg, walk);
                const int a_row = walk.mt * kMx4Tile, n0 = walk.nt * BN, wt = n0 / 128;
                const uint8_t* sa = p.sa + (int64_t)walk.mt * ktiles * kSfTile;
                const uint8_t* sw = p.sw + ((int64_t)q.expert * w_row_tiles + wt) * ktiles * kSfTile;
                const int boxes = (q.rows + p.box_rows - 1) / p.box_rows;
                const uint32_t a_bytes = boxes * p.box_rows * 128;
                for (int kb = 0; kb < num_kb; ++kb, s = (s + 1 == STAGES ? 0 : s + 1), phase ^= (s == 0)) {
                    mbar_wait_lean(&empty_bar[s], phase, dead, p.status);
                    const uint32_t sf = kSfTile * min(2, ktiles - 2 * kb);
                    mbar_expect_tx(&full_bar[s], a_bytes + S::kBBytes + 2 * sf);
                    uint8_t* a = smem + s * S::kStage;
                    uint8_t* b = a + kABytes;
                    uint8_t* f = b + S::kBBytes;
                    for (int i = 0; i < boxes; ++i) tma_load_2d(a + i * p.box_rows * 128, &map_a, &full_bar[s], kb * 128, a_row + i * p.box_rows);
                    tma_load_2d(b, &map_w, &full_bar[s], kb * 128, q.expert * p.N + n0);
                    bulk_load(f, sa + kb * 2 * kSfTile, sf, &full_bar[s]);
                    bulk_load(f + 2 * kSfTile, sw + kb * 2 * kSfTile, sf, &full_bar[s]);
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ scale bytes and products, one thread
        if (elect_one()) {
            const uint64_t da0 = smem_desc(smem_u32(smem), 16, 1024), db0 = smem_desc(smem_u32(smem + kABytes), 16, 1024);
            const uint64_t df0 = scale_desc(smem_u32(smem + kABytes + S::kBBytes));
            uint32_t stage = 0, phase = 0, local = 0;
            for (int t = first; t < last; t += step, ++local) {
                const uint32_t acc = local & 1, use = local >> 1;
                // a 64-column tile in the second half of W's row tile: its rows' bytes start two columns further
                const uint32_t shift = BN == 64 ? (uint32_t)((t % tiles_n) & 1) * 2 : 0;
                mbar_wait_lean(&tmem_empty_bar[acc], (use & 1) ^ 1, dead, p.status);
                tc_fence_after();
                const uint32_t d = tmem + acc * BN, fa = tmem + kSfCol, fw = fa + 8;
                for (int kb = 0; kb < num_kb; ++kb) {
                    mbar_wait_lean(&full_bar[stage], phase, dead, p.status);
                    tc_fence_after();
                    const uint64_t step = (uint64_t)stage * (S::kStage >> 4);
                    const uint64_t da = da0 + step, db = db0 + step, df = df0 + step;
                    const int cols = min(kSliceK, p.K - kb * kSliceK);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if (j * 128 >= cols) break;
                        copy_scales(fa + 4 * j, df + j * (kSfTile >> 4));
                        copy_scales(fw + 4 * j, df + (2 + j) * (kSfTile >> 4));
                    }
#pragma unroll
                    for (int kk = 0; kk < kSliceK / 64; ++kk) {
                        if (kk * 64 >= cols) break;
                        umma_mx4(d, da + kk * 2, db + kk * 2, instr_desc_mx4(BN, kk & 1), fa + 4 * (kk >> 1), fw + 4 * (kk >> 1) + shift,
                                 kb != 0 || kk != 0);
                    }
                    umma_commit(&empty_bar[stage]);
                    if (++stage == STAGES) { stage = 0; phase ^= 1; }
                }
                umma_commit(&tmem_full_bar[acc]);
            }
        }
    } else {
        // ------------------------------------------------------------------ epilogue: set `acc` drains accumulator `acc`
        const int quad = warp & 3, half = ((warp - 2) >> 2) & 1;
        const uint32_t acc = (uint32_t)(warp - 2) >> 3;
        Mx4Epilogue<OUT, S::kCols> epi(p, &map_c, boxes_c + (warp - 2) * S::kBox, lane);
        const uint32_t t_addr = tmem + acc * BN + ((uint32_t)(quad * 32) << 16) + half * S::kCols;
        uint32_t use = 0;
        Mx4Walk walk;
        walk.init(first + (int)acc * step, 2 * step, tiles_n);
        for (int t = first + (int)acc * step; t < last; t += 2 * step, walk.next(), ++use) {
            const Mx4Rows q = mx4_rows(p, seg, walk);
            mbar_wait_lean(&tmem_full_bar[acc], use & 1, dead, p.status);
            tc_fence_after();
            epi.begin(walk.nt * BN + half * S::kCols, q.c_row + quad * 32, q.rows - quad * 32, walk.mt * kMx4Tile + quad * 32);
#pragma unroll
            for (int c = 0; c < S::kCols / 32; ++c) {
                float v[32];
                tmem_load_32_nowait(t_addr + c * 32, (uint32_t*)v);
                tmem_load_wait();
                if (c == S::kCols / 32 - 1) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&tmem_empty_bar[acc]);
                }
                epi.chunk(c, v);
            }
            epi.end();
        }
        epi.finish();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
}

template <int BN, int STAGES, int OUT>
cudaError_t launch(const Mx4View& a, const Mx4View& w, Mx4Params p, int64_t max_tiles_m, cudaStream_t stream) {
    using S = Mx4Smem<BN, STAGES>;
    CUtensorMap ma, mw, mc;
    const uint64_t row = (uint64_t)p.K / 2;
    const uint64_t a_rows = a.offsets ? (uint64_t)a.capacity : (uint64_t)a.rows, w_rows = (uint64_t)w.rows * (w.E > 0 ? w.E : 1);
    p.box_rows = a.rows <= (p.offsets ? 96 * (int64_t)p.E : 96) ? 32 : 128;
    if (!make_map_u8(&ma, a.codes, row, a_rows, row, 128, p.box_rows, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_map_u8(&mw, w.codes, row, w_rows, row, 128, BN, CU_TENSOR_MAP_SWIZZLE_128B))
        return cudaErrorInvalidValue;
    // (few rows are written as they are: a tensor map takes half a microsecond of the host's time)
    p.tma_store = OUT <= OUT_BF16_ACT && p.M > 32 && tma_store_ok(p);
    mc = mw;
    if (p.tma_store && !make_map(&mc, p.C, (uint64_t)p.N, (uint64_t)p.M, (uint64_t)p.ldc, S::kCols, 32,
                                 S::kCols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B))
        return cudaErrorInvalidValue;
    static PerDeviceOnce once;
    auto kernel = gemm_mx4_kernel<BN, STAGES, OUT>;
    static_assert(S::bytes(kMaxExperts) <= 227 * 1024, "shared memory of a block");
    int dev;
    if (once.needed(&dev)) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::bytes(kMaxExperts));
        if (e != cudaSuccess) return e;
        once.mark(dev);
    }
    const int64_t tiles = max_tiles_m * ((p.N + BN - 1) / BN);
    const int sms = gemm_tc_sm_count();
    return launch_chained(kernel, (int)(tiles < sms ? tiles : sms), kThreadsMx4, S::bytes(p.offsets ? p.E : 0), stream, ma, mw, mc, p);
}

template <int BN, int STAGES>
cudaError_t launch_out(const Mx4View& a, const Mx4View& w, const Mx4Params& p, int dtype, int64_t max_tiles_m, cudaStream_t stream) {
    if (p.out_codes)
        return p.act == BIGMAC_ACT_GELU_ERF ? launch<BN, STAGES, OUT_MX4_GELU>(a, w, p, max_tiles_m, stream) : launch<BN, STAGES, OUT_MX4>(a, w, p, max_tiles_m, stream);
    if (dtype == BIGMAC_F32) return launch<BN, STAGES, OUT_F32>(a, w, p, max_tiles_m, stream);
    if (p.act == BIGMAC_ACT_IDENTITY) return launch<BN, STAGES, OUT_BF16>(a, w, p, max_tiles_m, stream);
    if (p.act == BIGMAC_ACT_GELU_ERF) return launch<BN, STAGES, OUT_BF16_GELU>(a, w, p, max_tiles_m, stream);
    return launch<BN, STAGES, OUT_BF16_ACT>(a, w, p, max_tiles_m, stream);
}

// Which tiles.  64 columns as long as every SM gets one tile at most: a CTA's loads are what few tiles wait for (one row, N 4096, K 4096 6.7 us
// against 7.0 with 128; 300 rows of N 4096, two rounds, 11.4 against 7.8).  CTA pairs for dense products of more than a round of 128 x 128
// tiles that are long enough for the pair's longer start and its single accumulator: us with 128 columns / pairs, t tiles of 128 x 128:
// t 256: K 512 4.9 / 5.8, K 1024 6.4 / 6.4, K 4096 12.8 / 10.1; t 512: K 256 6.5 / 6.6, K 512 7.2 / 7.0; t 1024: K 256 9.1 / 8.7; t 4096, K 4096
// 74 / 54.
int mx4_tile_of(const Mx4View& a, const Mx4View& w, int64_t tiles_m, int sms) {
    const int64_t tiles = tiles_m * ((w.rows + 127) / 128);
    if (tiles_m * ((w.rows + 63) / 64) <= sms) return 64;
    return !a.offsets && tiles > sms && tiles * a.K >= 1 << 18 ? 256 : 128;
}

}  // namespace

cudaError_t launch_mx4_matmul(const Mx4View& a, const Mx4View& w, int act, int dtype, void* c, int64_t ldc, const Mx4View* out, int* status,
                              cudaStream_t stream) {
    if (a.rows == 0 || w.rows == 0) return cudaSuccess;
    Mx4Params p{};
    if (out) { p.out_codes = out->codes; p.out_scales = out->scales; }
    p.C = c; p.ldc = ldc; p.sa = a.scales; p.sw = w.scales; p.offsets = a.offsets;
    p.M = a.rows; p.N = w.rows; p.K = a.K; p.E = a.E; p.capacity = a.capacity;
    p.act = act; p.status = status;
    const int64_t tiles_m = a.offsets ? a.capacity / kMx4Tile : (a.rows + kMx4Tile - 1) / kMx4Tile;
    const int sms = gemm_tc_sm_count();
    int tile = switches().mx4_tile;
    if (tile != 64 && tile != 128 && (tile != 256 || a.offsets)) tile = mx4_tile_of(a, w, tiles_m, sms);
    if (tile == 256) return launch_mx4_matmul_pair(a, w, p, dtype, stream);
    return tile == 64 ? launch_out<64, 6>(a, w, p, dtype, tiles_m, stream) : launch_out<128, 4>(a, w, p, dtype, tiles_m, stream);
}

}  // namespace bigmac
