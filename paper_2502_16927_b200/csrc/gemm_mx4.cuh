// Pieces that the products of microscaled 4-bit matrices share: instructions, the activation, what leaves a tile and how.
#pragma once
#include "tc_pair.cuh"
#include "mx4.h"

namespace bigmac {
namespace mx4 {

using namespace tc;

constexpr int kSliceK = 256;                               // columns of a stage: one 128-byte row of codes
constexpr uint32_t kABytes = 128 * 128;
constexpr uint32_t kSfTile = 512;
constexpr int kEpi = 16;                                   // epilogue warps, two sets with two to a lane quadrant
constexpr int kThreadsMx4 = (2 + kEpi) * 32;

struct Mx4Params {
    void* C;
    int64_t ldc;
    const uint8_t *sa, *sw;                                // scale bytes
    uint8_t *out_codes, *out_scales;                       // OUT_MX4: the result's
    const int32_t* offsets;                                // grouped: the caller's table
    int M, N, K, E;
    int64_t capacity;                                      // rows that A has room for (grouped)
    int act, tma_store;
    int box_rows;                                          // of A's codes: a tile with few rows loads few
    int* status;
};

// May rows of bf16 leave by TMA?  Rows on 16-byte boundaries, and whole 16 bytes of columns: a store that the tensor map cuts off inside a
// 16-byte piece writes the rest of the piece, too, which belongs to whoever has the columns behind C.
inline bool tma_store_ok(const Mx4Params& p) { return p.ldc % 8 == 0 && p.N % 8 == 0 && (uintptr_t)p.C % 16 == 0; }

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
// 512 bytes of scales, 32 rows of 16 bytes, to four columns of tensor memory in all four lane quadrants.
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
// Without swizzle: groups of 8 rows of 16 bytes, 128 bytes apart.
__device__ __forceinline__ uint64_t scale_desc(uint32_t addr) {
    return (uint64_t)((addr & 0x3ffff) >> 4) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46);
}
__device__ __forceinline__ void umma_mx4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
}
// Instruction descriptor: e2m1 x e2m1, scales ue8m0, M 128, N bn; `half`: which two of a column's four scale bytes.
__host__ __device__ constexpr uint32_t instr_desc_mx4(int bn, int half) {
    return ((uint32_t)(2 * half) << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(bn >> 3) << 17) | (1u << 23) | ((uint32_t)(128 >> 4) << 24) |
           ((uint32_t)(2 * half) << 29);
}

// GELU of 32 accumulators for an output in bf16 or 4 bits:  z Phi(z) = |z| ((z > 0) - q),  q = Phi(-|z|) = 2^P(|z|).  P is the minimax fit of
// log2 Phi(-x) on [0, 14] (linear program on Chebyshev nodes, the error behind 8 allowed to be ten times that up to 5), of odd degree with a negative
// leading coefficient: behind 14 it falls on to minus infinity, so q is 0 there without a look at the argument.  An error of P is a relative
// one of q, so the negative tail, whose values are the scales and codes of 4-bit blocks that hold nothing else, is as good as the rest: evaluated in fp32, z Phi(z) is off
// by 1.0e-5 of itself up to |z| = 5 and by 1.1e-4 behind it (a bf16 half step is 2^-9 to 2^-8); q below 2^-126 (z < -13) becomes 0.  Infinities are
// those of the definition: z = inf gives inf, -inf the product with 0, a NaN.  131072 rows of r 256, h 1024: 82.5 us; without an activation 54; with a saturating
// polynomial for Phi itself, which is off by up to 3.7e-5 whatever the size of the value (a fifth of it at z = -4, all of it from -4.3 on), 78; erff 142.
__device__ __forceinline__ void gelu_chunk(float* v) {
    constexpr float kC[10] = {-1.0000075101852417f, -1.1512371301651f, -0.4582904577255249f, -0.054337747395038605f, 0.008810615167021751f,
                              -0.0010507769184187055f, 8.72075543156825e-05f, -4.706160325440578e-06f, 1.4724672325883148e-07f, -2.0163450908938785e-09f};
    constexpr int kG = 8;                                  // pairs side by side, so that no multiply-add waits for the one before
#pragma unroll
    for (int g = 0; g < 16; g += kG) {
        f32x2_t x[kG], P[kG];
#pragma unroll
        for (int i = 0; i < kG; ++i) {
            x[i] = pk2(fabsf(v[2 * (g + i)]), fabsf(v[2 * (g + i) + 1]));
            P[i] = fma2(pk2(kC[9], kC[9]), x[i], pk2(kC[8], kC[8]));
        }
#pragma unroll
        for (int k = 7; k >= 0; --k)
#pragma unroll
            for (int i = 0; i < kG; ++i) P[i] = fma2(P[i], x[i], pk2(kC[k], kC[k]));
#pragma unroll
        for (int i = 0; i < kG; ++i) {
            float &z0 = v[2 * (g + i)], &z1 = v[2 * (g + i) + 1], p0, p1;
            upk2(P[i], p0, p1);
            const float c0 = (z0 > 0.0f ? 1.0f : 0.0f) - fast_ex2(p0), c1 = (z1 > 0.0f ? 1.0f : 0.0f) - fast_ex2(p1);
            upk2(mul2(x[i], pk2(c0, c1)), z0, z1);
        }
    }
}

// GELU of 32 accumulators for an output in fp32: as above with q = exp(-z^2 / 2) G(|z|), G(x) = erfcx(x / sqrt 2) / 2 as a polynomial in t = 1 / (1 + 0.3 x), its
// minimax fit in relative error (5.7e-8) on [0, 13.3].  Off by four units of 2^-23 near 0 and, with the exponent's rounding, by z^2 / 2 of them far
// from it.  (1 + erf, whose negative tail is a difference of two numbers near 1, is off by 6e-8 of |z| whatever the value: a tenth of it at z = -5.)
__device__ __forceinline__ void gelu_chunk_f32(float* v) {
    constexpr float kC[9] = {6.6862244239018764e-06f, 0.11949588358402252f, 0.121862031519413f, 0.0949108824133873f, 0.1420028954744339f,
                             -0.07573675364255905f, 0.22798816859722137f, -0.16884131729602814f, 0.03831155598163605f};
    constexpr int kG = 4;
#pragma unroll
    for (int g = 0; g < 16; g += kG) {
        f32x2_t x[kG], t[kG], P[kG];
#pragma unroll
        for (int i = 0; i < kG; ++i) {
            x[i] = pk2(fabsf(v[2 * (g + i)]), fabsf(v[2 * (g + i) + 1]));
            float d0, d1;
            upk2(fma2(x[i], pk2(0.3f, 0.3f), pk2(1.0f, 1.0f)), d0, d1);
            t[i] = pk2(fast_rcp(d0), fast_rcp(d1));
            P[i] = fma2(pk2(kC[8], kC[8]), t[i], pk2(kC[7], kC[7]));
        }
#pragma unroll
        for (int k = 6; k >= 0; --k)
#pragma unroll
            for (int i = 0; i < kG; ++i) P[i] = fma2(P[i], t[i], pk2(kC[k], kC[k]));
#pragma unroll
        for (int i = 0; i < kG; ++i) {
            float &z0 = v[2 * (g + i)], &z1 = v[2 * (g + i) + 1], e0, e1, q0, q1;
            upk2(mul2(mul2(x[i], pk2(-0.72134752044448170f, -0.72134752044448170f)), x[i]), e0, e1);
            upk2(mul2(pk2(fast_ex2(e0), fast_ex2(e1)), P[i]), q0, q1);
            upk2(mul2(x[i], pk2((z0 > 0.0f ? 1.0f : 0.0f) - q0, (z1 > 0.0f ? 1.0f : 0.0f) - q1)), z0, z1);
        }
    }
}
// GELU's tanh form, z (1 + tanh w) / 2 = z / (1 + exp(-2 w)), which has no such difference; -2 w / ln 2 = z (a + b z^2).
__device__ __forceinline__ void gelu_tanh_chunk(float* v) {
    constexpr float kA = -2.3022081986f, kB = -0.1029432396f;             // -2 sqrt(2 / pi) / ln 2, and 0.044715 of it
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const f32x2_t z = pk2(v[2 * i], v[2 * i + 1]);
        float e0, e1;
        upk2(mul2(z, fma2(mul2(z, z), pk2(kB, kB), pk2(kA, kA))), e0, e1);
        upk2(mul2(z, pk2(fast_rcp(1.0f + fast_ex2(e0)), fast_rcp(1.0f + fast_ex2(e1)))), v[2 * i], v[2 * i + 1]);
    }
}
// The activation of a chunk, chosen once for 32 elements (for each of them: ReLU of 131072 x 1024 bf16 results 90 us, so 54); the erf form of narrow results
// has kernels of its own.
template <bool ERF>
__device__ __forceinline__ void act_chunk(int act, float* v) {
    if (ERF && act == BIGMAC_ACT_GELU_ERF) gelu_chunk_f32(v);
    else if (act == BIGMAC_ACT_GELU_TANH) gelu_tanh_chunk(v);
    else if (act == BIGMAC_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = act_apply(BIGMAC_ACT_RELU, v[i]);
    }
}

// The tiles of a walker: t, t + step, ...  All columns of a row tile follow each other (its codes stay in L2).
struct Mx4Walk {
    int mt, nt, e, step_m, step_n, tiles_n;
    __device__ __forceinline__ void init(int t, int step, int n) {
        tiles_n = n;
        mt = t / n; nt = t - mt * n;
        step_m = step / n; step_n = step - step_m * n;
        e = -1;
    }
    __device__ __forceinline__ void next() {
        mt += step_m; nt += step_n;
        if (nt >= tiles_n) { nt -= tiles_n; ++mt; }
    }
    // The expert of row tile mt, which never falls from tile to tile.
    __device__ __forceinline__ int expert(const Mx4Segments& seg) {
        if (e < 0) e = mx4_find(seg.tiles, seg.E, mt);
        while (e + 1 < seg.E && seg.tiles[e + 1] <= mt) ++e;
        return e;
    }
};
struct Mx4Rows {
    int expert, c_row, rows;                               // first row in C, rows of this tile that exist
};
__device__ __forceinline__ Mx4Rows mx4_rows(const Mx4Params& p, const Mx4Segments& seg, Mx4Walk& w) {
    if (!p.offsets) return {0, w.mt * kMx4Tile, min(kMx4Tile, p.M - w.mt * kMx4Tile)};
    const int e = w.expert(seg), within = (w.mt - seg.tiles[e]) * kMx4Tile;
    return {e, seg.offsets[e] + within, min(kMx4Tile, seg.count(e) - within)};
}

// 32 columns of a row, packed, to the warp's box of 32 rows by COLS columns, laid out for a TMA store with the swizzle of its row's width.
template <int COLS>
__device__ __forceinline__ void stage_row(uint8_t* box, int lane, int chunk, const uint32_t* w) {
    if (COLS == 64) {
        uint8_t* row = box + lane * 128;
#pragma unroll
        for (int j = 0; j < 4; ++j) st_shared_16B(row + (((chunk * 4 + j) ^ (lane & 7)) << 4), w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
    } else {
        stage_row_bf16(box, lane, w);
    }
}

// 32 columns of a row are a block of the result in 4 bits: its scale and codes from the fp32 numbers, without a rounding between.
__device__ __forceinline__ void store_block(const Mx4Params& p, float* v, int row, int block) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) top = max_nan(top, fabsf(v[i]));
    const uint32_t s = mx4_scale_byte(top);
    uint32_t c[4] = {0u, 0u, 0u, 0u};
    if (s != 255u) {
        const f32x2_t factor = mx4_factor2(s);
#pragma unroll
        for (int i = 0; i < 16; ++i) upk2(mul2(pk2(v[2 * i], v[2 * i + 1]), factor), v[2 * i], v[2 * i + 1]);
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = mx4_e2m1x8(v + 8 * i);
    }
    *(uint4*)(p.out_codes + (int64_t)row * (p.N / 2) + block * 16) = make_uint4(c[0], c[1], c[2], c[3]);
    uint8_t* at = p.out_scales + mx4_scale_at(row, block, mx4_ktiles(p.N));
    *at = (uint8_t)s;
    if (block + 1 == p.N / 32)
        for (int b = block + 1; b & 3; ++b) *++at = 0;                   // behind the last block of the row
}

// What the epilogue does is fixed at compile time: with every way in one kernel its warps waited for instructions.
enum { OUT_BF16 = 0, OUT_BF16_GELU, OUT_BF16_ACT, OUT_F32, OUT_MX4_GELU, OUT_MX4 };
__host__ __device__ constexpr bool is_mx4_out(int out) { return out == OUT_MX4 || out == OUT_MX4_GELU; }

// What an epilogue warp does with its 32 rows and COLS columns of a finished tile: 32 columns (a chunk) after each other.
template <int OUT, int COLS>
struct Mx4Epilogue {
    static constexpr int kChunks = COLS / 32;
    static constexpr uint32_t kBox = 32 * COLS * 2;
    const Mx4Params& p;
    const CUtensorMap* map_c;
    uint8_t* box;
    int lane;
    bool vec_ok;
    // the tile's
    int first_col, row0, rows, a_row0;                     // column, first of the warp's rows in C, how many exist, their place in A
    bool by_tma, by_rows;

    __device__ __forceinline__ Mx4Epilogue(const Mx4Params& p_, const CUtensorMap* map, uint8_t* box_, int lane_) : p(p_), map_c(map), box(box_), lane(lane_) {
        constexpr int esz = OUT == OUT_F32 ? 4 : 2;
        vec_ok = (p.ldc * esz) % 32 == 0 && (uintptr_t)p.C % 32 == 0;
    }
    // Whole boxes leave by TMA (a dense C is cut off by the tensor map), the last rows of a segment row by row, rows that are not on 16-byte boundaries
    // through the box, too, a row after the other (lanes that each wrote their own row element by element took 20 times as long).
    __device__ __forceinline__ void begin(int first_col_, int row0_, int rows_, int a_row0_) {
        first_col = first_col_; row0 = row0_; rows = rows_; a_row0 = a_row0_;
        by_tma = OUT <= OUT_BF16_ACT && p.tma_store && (rows >= 32 || !p.offsets);
        by_rows = OUT <= OUT_BF16_ACT && !by_tma && !vec_ok;
        if (OUT <= OUT_BF16_ACT) {
            if (elect_one()) tma_store_wait_read();        // the box before has left shared memory
            __syncwarp();
        }
    }
    __device__ __forceinline__ void chunk(int c, float* v) {
        const int col0 = first_col + c * 32;
        if (col0 >= p.N || rows <= 0) return;              // nothing of the tile is here: a warp's 32 rows may lie behind a segment's last
        if (OUT == OUT_BF16_GELU || OUT == OUT_MX4_GELU) {
            gelu_chunk(v);
        } else if (OUT != OUT_BF16 && p.act != BIGMAC_ACT_IDENTITY) {
            act_chunk<OUT == OUT_F32>(p.act, v);
        }
        if constexpr (is_mx4_out(OUT)) {
            if (lane < rows) store_block(p, v, a_row0 + lane, col0 / 32);
        } else if constexpr (OUT == OUT_F32) {
            if (lane >= rows) return;
            float* to = (float*)p.C + (int64_t)(row0 + lane) * p.ldc + col0;
            if (vec_ok && col0 + 32 <= p.N) {
#pragma unroll
                for (int i = 0; i < 4; ++i) st_global_32B(to + 8 * i, (const uint32_t*)v + 8 * i);
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (col0 + i < p.N) to[i] = v[i];
            }
        } else {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
            if (by_tma || by_rows) {
                stage_row<COLS>(box, lane, c, w);
            } else if (lane < rows) {
                __nv_bfloat16* to = (__nv_bfloat16*)p.C + (int64_t)(row0 + lane) * p.ldc + col0;
                if (col0 + 32 <= p.N) {
                    st_global_32B(to, w);
                    st_global_32B(to + 16, w + 8);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (col0 + i < p.N) ((uint16_t*)to)[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
                }
            }
        }
    }
    __device__ __forceinline__ void end() {
        if (OUT > OUT_BF16_ACT || first_col >= p.N || rows <= 0) return;
        if (by_tma) {
            fence_async_smem();
            __syncwarp();
            if (elect_one()) {
                tma_store_2d(map_c, box, first_col, row0);
                tma_store_commit();
            }
        } else if (by_rows) {
            __syncwarp();
            constexpr int kAtOnce = 64 / COLS;             // rows that 32 lanes with two columns each cover
            const int sub = kAtOnce == 2 ? lane >> 4 : 0, pair = kAtOnce == 2 ? lane & 15 : lane;
            const bool words = p.ldc % 2 == 0 && (uintptr_t)p.C % 4 == 0;
            const int n = min(rows, 32), col = first_col + 2 * pair;
            for (int r = sub; r < n; r += kAtOnce) {
                const int piece = COLS == 64 ? (pair >> 2) ^ (r & 7) : (pair >> 2) ^ ((r >> 1) & 3);
                const uint32_t w = *(const uint32_t*)(box + r * COLS * 2 + piece * 16 + (pair & 3) * 4);
                uint16_t* to = (uint16_t*)p.C + (int64_t)(row0 + r) * p.ldc + col;
                if (words && col + 2 <= p.N) {
                    *(uint32_t*)to = w;
                } else {
                    if (col < p.N) to[0] = (uint16_t)w;
                    if (col + 1 < p.N) to[1] = (uint16_t)(w >> 16);
                }
            }
            __syncwarp();                                  // the box is read: the next tile's rows may go in
        }
    }
    __device__ __forceinline__ void finish() {
        if (OUT <= OUT_BF16_ACT && elect_one()) tma_store_wait_read();   // the boxes have left shared memory; the writes land before the grid ends
    }
};

}  // namespace mx4

// Dense products of many 256 x 256 tiles (gemm_mx4_pair.cu).
cudaError_t launch_mx4_matmul_pair(const Mx4View& a, const Mx4View& w, const mx4::Mx4Params& p, int dtype, cudaStream_t stream);

}  // namespace bigmac
