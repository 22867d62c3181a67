// Shared by the units that work on microscaled 4-bit matrices: the layout of a matrix and of the segments of a grouped one.
//
// A matrix of `rows` rows and K columns (K a multiple of 32): element (m, k) is a 4-bit float (e2m1) in nibble k % 2 of byte k / 2
// of row m, times 2^(s - 127) with s the scale byte of its block of 32 columns.  Scale bytes lie as tcgen05.cp moves them to tensor memory, in tiles of
// 128 rows by 4 blocks (128 columns): tile (m / 128, k / 128) is 512 consecutive bytes, in it byte (m % 32) 16 + (m / 32 % 4) 4 +
// (k / 32 % 4); tiles of one row tile follow each other.
// A grouped matrix holds the segments of E experts, each from a multiple of 128 rows on.
#pragma once
#include "internal.h"

namespace bigmac {

constexpr int kMx4Tile = 128;

__host__ __device__ inline int mx4_ktiles(int K) { return (K + 127) / 128; }
__host__ __device__ inline int64_t mx4_scale_at(int64_t row, int block, int ktiles) {
    return ((row >> 7) * ktiles + (block >> 2)) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}
// Rows a grouped matrix has room for: every expert may fill its last 128 rows with one row only.
inline int64_t mx4_padded_rows(int64_t rows, int E) {
    const int64_t ragged = rows < E ? rows : E;
    return (rows + ragged * (kMx4Tile - 1)) / kMx4Tile * kMx4Tile;
}

#ifdef __CUDACC__
// The segments of a grouped matrix in shared memory, 2 E + 2 words: the caller's table cut to [0, rows], so that a table that is none reads and
// writes nothing outside, and the row tiles before every expert.  All threads of a block call it.
struct Mx4Segments {
    const int32_t *offsets, *tiles;    // [E + 1] each
    int E;
    __device__ __forceinline__ void load(int32_t* smem, const int32_t* __restrict__ table, int E_, int rows) {
        int32_t* cut = smem;
        int32_t* before = smem + E_ + 1;
        offsets = cut; tiles = before; E = E_;
        for (int e = threadIdx.x; e <= E; e += blockDim.x) cut[e] = min(max(table[e], 0), rows);
        __syncthreads();
        if (threadIdx.x < 32) {
            const int lane = threadIdx.x, per = (E + 31) / 32, e0 = min(E, lane * per), e1 = min(E, e0 + per);
            int mine = 0;
            for (int e = e0; e < e1; ++e) mine += tiles_of(e);
            mine = min(mine, 1 << 25);                 // twice what memory has room for: the sum over a table that is none stays in 32 bits
            int run = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int a = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += a;
            }
            if (lane == 31) before[E] = run;
            run -= mine;
            for (int e = e0; e < e1; ++e) { before[e] = run; run += tiles_of(e); }
        }
        __syncthreads();
    }
    __device__ __forceinline__ int count(int e) const { return max(offsets[e + 1] - offsets[e], 0); }
    __device__ __forceinline__ int tiles_of(int e) const { return (count(e) + kMx4Tile - 1) / kMx4Tile; }
};
// The last e in [0, E) with table[e] <= v; table ascending, table[0] <= v.
__device__ __forceinline__ int mx4_find(const int32_t* table, int E, int v) {
    int lo = 0, hi = E - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (table[mid] <= v) lo = mid; else hi = mid - 1;
    }
    return lo;
}
// Eight values to four bytes of codes.
__device__ __forceinline__ uint32_t mx4_e2m1x8(const float* v) {
    uint32_t out;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(out) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return out;
}
__device__ __forceinline__ float max_nan(float a, float b) { float d; asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b)); return d; }
// The scale byte of a block whose largest magnitude is `top` (a NaN if it has one).
__device__ __forceinline__ uint32_t mx4_scale_byte(float top) {
    const uint32_t bits = __float_as_uint(top);
    return bits < 0x7f800000u ? (uint32_t)max((int)(bits >> 23) - 2, 0) : 255u;
}
// The factor 2^(127 - s), twice, as a pair of fp32 numbers.
__device__ __forceinline__ unsigned long long mx4_factor2(uint32_t s) {
    const unsigned long long f = (unsigned long long)(254u - s) << 23;
    return f | f << 32;
}
#endif

struct Mx4View {                      // one matrix, or E stacked ones (weights), or the segments of E experts (offsets set)
    uint8_t *codes, *scales;
    int rows, K, E;                   // rows of the caller's order (of one matrix, where E are stacked)
    const int32_t* offsets;
    int64_t capacity;                 // rows that `codes` and `scales` have room for
};

cudaError_t launch_mx4_quantize(const void* x, int dtype, int64_t ld, const int32_t* slot_of_row, int k, int x_rows, const Mx4View& out,
                                cudaStream_t stream);
cudaError_t launch_mx4_dequantize(const Mx4View& q, void* y, int dtype, int64_t ld, cudaStream_t stream);
// act(a w^T) to c (bf16 or fp32) or, with `out`, to a matrix in 4 bits with a's rows (c, dtype unused).
cudaError_t launch_mx4_matmul(const Mx4View& a, const Mx4View& w, int act, int dtype, void* c, int64_t ldc, const Mx4View* out, int* status,
                              cudaStream_t stream);

}  // namespace bigmac
