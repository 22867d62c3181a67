// Rows to microscaled 4-bit floating point and back (layout: mx4.h).
//
//   amax = max |x| over a block of 32 columns;  s = max(0, floor(log2 amax) - 2 + 127);  code = e2m1(x 2^(127 - s))
//
// The scale is the power of two that brings the block's largest magnitude into [4, 8); e2m1 holds 0 0.5 1 1.5 2 3 4 6 and their
// negatives, rounding to the nearest (ties to the even code), magnitudes above 6 become 6.  x 2^(127 - s) is a product with a
// power of two, so exact but for results that underflow, which are far below 0.25 and become 0: a code depends on nothing but its block.
// A block with an infinity or a NaN has scale byte 255 (NaN) and zero codes, and every product with it is NaN.
//
// Bound by memory: 2 bytes (bf16) in, 17/32 out per element.  A thread takes 16 columns (two 16-byte loads, 8 bytes of codes), two
// threads a block, eight a word of scale bytes; a row goes to as many lanes as it has 16-column pieces, up to a warp.
#include "mx4.h"

namespace bigmac {

namespace {

constexpr unsigned kAll = 0xffffffffu;
constexpr int kThreads = 256;

// Where row i of the caller's order lies in the matrix; -1: in no segment.
struct RowMap {
    const int32_t* first;             // [E] of the caller's order, shared memory
    const int32_t* tiles;             // [E + 1]
    const int32_t* end;               // [E]
    int E;
    int64_t capacity;
    __device__ __forceinline__ int64_t at(int i) const {
        if (E == 0) return i;
        const int e = mx4_find(first, E, i);
        const int64_t row = (int64_t)tiles[e] * kMx4Tile + (i - first[e]);
        return i >= first[e] && i < end[e] && row < capacity ? row : -1;
    }
};

__device__ __forceinline__ RowMap load_map(const Mx4View& q, int32_t* smem) {
    RowMap m{smem, smem + q.E, smem + 2 * q.E + 1, q.offsets ? q.E : 0, q.capacity};
    if (m.E) {
        for (int e = threadIdx.x; e < q.E; e += blockDim.x) {
            const Mx4Segment s = mx4_segment(q.offsets, e, q.rows);
            smem[e] = s.first;
            smem[2 * q.E + 1 + e] = s.first + s.count;
        }
        if (threadIdx.x < 32) mx4_tile_prefix(q.offsets, q.E, q.rows, smem + q.E);
        __syncthreads();
    }
    return m;
}

// Eight values to four bytes of codes.
__device__ __forceinline__ uint32_t e2m1x8(const float* v) {
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

__device__ __forceinline__ void load16(const __nv_bfloat16* p, float* v) {
    uint4 a = __ldg((const uint4*)p), b = __ldg((const uint4*)p + 1);
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void load16(const float* p, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 a = __ldg((const float4*)p + i);
        v[4 * i] = a.x; v[4 * i + 1] = a.y; v[4 * i + 2] = a.z; v[4 * i + 3] = a.w;
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) mx4_quantize_kernel(const T* __restrict__ x, int64_t ld, const int32_t* __restrict__ slot_of_row,
                                                                int k, int64_t x_slots, Mx4View q, int lanes_log2) {
    extern __shared__ int32_t smem[];
    grid_dependency_launch();
    grid_dependency_wait();
    const RowMap map = load_map(q, smem);
    const int pieces = q.K / 16, ktiles = mx4_ktiles(q.K), lanes = 1 << lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int per_block = kThreads >> lanes_log2;
    const int64_t stride = (int64_t)gridDim.x * per_block;
    for (int64_t base = (int64_t)blockIdx.x * per_block; base < q.rows; base += stride) {     // the same trips for a whole block
        const int64_t i = base + (threadIdx.x >> lanes_log2);
        const int64_t row = i < q.rows ? map.at((int)i) : -1;
        int64_t src = i;
        if (row >= 0 && slot_of_row) {
            const int slot = slot_of_row[i];
            src = slot >= 0 && slot < x_slots ? slot / k : -1;          // a slot that is none: a row of zeros
        }
        for (int p0 = 0; p0 < pieces; p0 += lanes) {
            const int p = p0 + lane;
            float v[16];
            uint32_t top = 0;
            const bool mine = row >= 0 && p < pieces;
            if (mine && src >= 0) {
                load16(x + src * ld + p * 16, v);
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = 0.0f;
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
            top = max(top, __shfl_xor_sync(kAll, top, 1));
            const bool finite = top < 0x7f800000u;
            const uint32_t s = finite ? (uint32_t)max((int)(top >> 23) - 2, 0) : 255u;
            const float inverse = __uint_as_float((finite ? 254u - s : 0u) << 23);
            uint2 codes = make_uint2(0u, 0u);
            if (finite) {
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] *= inverse;
                codes = make_uint2(e2m1x8(v), e2m1x8(v + 8));
            }
            // four blocks, eight lanes: one word of scale bytes (zero behind the last block of the row)
            uint32_t word = mine ? s << (8 * ((p >> 1) & 3)) : 0u;
            word |= __shfl_xor_sync(kAll, word, 2);
            word |= __shfl_xor_sync(kAll, word, 4);
            if (mine) {
                *(uint2*)(q.codes + row * (q.K / 2) + p * 8) = codes;
                if ((p & 7) == 0) *(uint32_t*)(q.scales + mx4_scale_at(row, p >> 1, ktiles)) = word;
            }
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) mx4_dequantize_kernel(Mx4View q, T* __restrict__ y, int64_t ld, int lanes_log2) {
    extern __shared__ int32_t smem[];
    grid_dependency_launch();
    grid_dependency_wait();
    const RowMap map = load_map(q, smem);
    const int pieces = q.K / 16, ktiles = mx4_ktiles(q.K), lanes = 1 << lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int per_block = kThreads >> lanes_log2;
    const int64_t stride = (int64_t)gridDim.x * per_block;
    for (int64_t i = (int64_t)blockIdx.x * per_block + (threadIdx.x >> lanes_log2); i < q.rows; i += stride) {
        const int64_t row = map.at((int)i);
        if (row < 0) continue;
        for (int p = lane; p < pieces; p += lanes) {
            const uint2 c = __ldg((const uint2*)(q.codes + row * (q.K / 2) + p * 8));
            const uint32_t s = __ldg(q.scales + mx4_scale_at(row, p >> 1, ktiles));
            // 2^(s - 127): a subnormal for 0, a NaN for 255
            const float scale = __uint_as_float(s == 255u ? 0x7fffffffu : s ? s << 23 : 0x00400000u);
            float v[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const uint32_t n = ((j < 8 ? c.x : c.y) >> (4 * (j & 7))) & 15u, m = n & 7u;
                // codes 2 to 7: two bits of exponent, one of mantissa; 0 and 1: 0 and 0.5
                const float mag = m < 2u ? 0.5f * (float)m : __uint_as_float((m + 252u) << 22);
                v[j] = __uint_as_float(__float_as_uint(mag) | ((n & 8u) << 28)) * scale;
            }
            T* out = y + i * ld + p * 16;
            if constexpr (sizeof(T) == 2) {
                uint32_t w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);      // exact: two bits, the exponents of fp32
                    w[j] = *reinterpret_cast<uint32_t*>(&b);
                }
                ((uint4*)out)[0] = make_uint4(w[0], w[1], w[2], w[3]);
                ((uint4*)out)[1] = make_uint4(w[4], w[5], w[6], w[7]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) ((float4*)out)[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
            }
        }
    }
}

int lanes_log2_of(int K) {
    int l = 3;                         // eight lanes put a word of scale bytes together
    while (l < 5 && (1 << l) < K / 16) ++l;
    return l;
}
int grid_of(int64_t rows, int lanes_log2) {
    const int64_t per_block = kThreads >> lanes_log2, want = (rows + per_block - 1) / per_block;
    const int64_t most = (int64_t)gemm_tc_sm_count() * 8;               // 2048 threads on every SM
    return (int)(want < most ? want : most);
}
size_t map_bytes(const Mx4View& q) { return q.offsets ? (size_t)(3 * q.E + 1) * 4 : 0; }

}  // namespace

cudaError_t launch_mx4_quantize(const void* x, int dtype, int64_t ld, const int32_t* slot_of_row, int k, int x_rows, const Mx4View& q,
                                cudaStream_t stream) {
    if (q.rows == 0) return cudaSuccess;
    const int l = lanes_log2_of(q.K), grid = grid_of(q.rows, l);
    const int64_t slots = (int64_t)x_rows * k;
    if (dtype == BIGMAC_BF16)
        return launch_chained(mx4_quantize_kernel<__nv_bfloat16>, grid, kThreads, map_bytes(q), stream, (const __nv_bfloat16*)x, ld, slot_of_row, k,
                              slots, q, l);
    return launch_chained(mx4_quantize_kernel<float>, grid, kThreads, map_bytes(q), stream, (const float*)x, ld, slot_of_row, k, slots, q, l);
}

cudaError_t launch_mx4_dequantize(const Mx4View& q, void* y, int dtype, int64_t ld, cudaStream_t stream) {
    if (q.rows == 0) return cudaSuccess;
    const int l = lanes_log2_of(q.K), grid = grid_of(q.rows, l);
    if (dtype == BIGMAC_BF16)
        return launch_chained(mx4_dequantize_kernel<__nv_bfloat16>, grid, kThreads, map_bytes(q), stream, q, (__nv_bfloat16*)y, ld, l);
    return launch_chained(mx4_dequantize_kernel<float>, grid, kThreads, map_bytes(q), stream, q, (float*)y, ld, l);
}

}  // namespace bigmac
