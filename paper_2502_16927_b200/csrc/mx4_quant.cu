// Rows to microscaled 4-bit floating point and back (layout: mx4.h).
//
//   amax = max |x| over a block of 32 columns;  s = max(0, floor(log2 amax) - 2 + 127);  code = e2m1(x 2^(127 - s))
//
// The scale is the power of two that brings the block's largest magnitude into [4, 8); e2m1 holds 0 0.5 1 1.5 2 3 4 6 and their
// negatives, rounding to the nearest (ties to the even code), magnitudes above 6 become 6.  x 2^(127 - s) is a product with a
// power of two, so exact but for results that underflow, which are far below 0.25 and become 0: a code depends on nothing but its block.
// A block with an infinity or a NaN has scale byte 255 (NaN) and zero codes, and every product with it is NaN.
//
// Bound by memory (2 bytes (bf16) in, 17/32 out per element) and, close to it, by instructions: a thread takes a whole block (64 bytes of bf16, 16 of
// codes), so that scale and places are worked out once for it; with half a block a thread 16384 rows of 4096 took 37 us, now 34.  Four
// threads put a word of scale bytes together; a row goes to as many lanes as it has blocks, up to a warp.  A warp has a chunk of rows, whose
// places and sources its lanes look up at once, a row each: done by every lane of a row they were half of the instructions of a gathered row of 256.
#include "mx4.h"

namespace bigmac {

namespace {

constexpr unsigned kAll = 0xffffffffu;
constexpr int kThreads = 256;

// Where row i of the caller's order lies in the matrix; -1: in no segment.
struct RowMap {
    Mx4Segments seg;
    int64_t capacity;
    __device__ __forceinline__ RowMap(const Mx4View& q, int32_t* smem) : capacity(q.capacity) {
        seg.E = 0;
        if (q.offsets) seg.load(smem, q.offsets, q.E, q.rows);
    }
    __device__ __forceinline__ int at(int i) const {
        if (seg.E == 0) return i;
        const int e = mx4_find(seg.offsets, seg.E, i), within = i - seg.offsets[e];
        const int64_t row = (int64_t)seg.tiles[e] * kMx4Tile + within;
        return within >= 0 && within < seg.count(e) && row < capacity ? (int)row : -1;
    }
};

// The work is cut into units: up to 1024 columns (a warp's 32 a lane) of a row.  A warp takes chunks of 32 units at most, one after the other over the
// grid, a pass of as many units as its lanes have room for at a time.
struct Chunks {
    int lane, group, per_pass, chunk, segments;
    int64_t units, first, step;
    __device__ __forceinline__ Chunks(int64_t rows, int K, int lanes_log2, int chunk_) {
        per_pass = 32 >> lanes_log2; chunk = chunk_;
        lane = threadIdx.x & ((1 << lanes_log2) - 1); group = (threadIdx.x & 31) >> lanes_log2;
        segments = (K + 1023) / 1024;
        units = rows * segments;
        const int warps = blockDim.x >> 5;
        first = ((int64_t)blockIdx.x * warps + (threadIdx.x >> 5)) * chunk;
        step = (int64_t)gridDim.x * warps * chunk;
    }
    // The row of a unit and its first block.
    __device__ __forceinline__ int row_of(int64_t unit, int& block) const {
        int row;
        if (segments == 1) row = (int)unit;
        else if (units <= 0xffffffffll) row = (int)((uint32_t)unit / (uint32_t)segments);     // a fifth of a 64-bit division
        else row = (int)(unit / segments);
        block = (int)(unit - (int64_t)row * segments) * 32;
        return row;
    }
};

// A block's 32 elements as they lie in memory; their largest magnitude (a NaN if there is one); the codes of their products with a power of two.
template <typename T>
struct Block {
    static constexpr int kWords = 8 * sizeof(T);
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T* p, bool by32) {
        if (by32) {
#pragma unroll
            for (int i = 0; i < kWords / 8; ++i)
                asm volatile("ld.global.nc.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                             : "=r"(w[8 * i]), "=r"(w[8 * i + 1]), "=r"(w[8 * i + 2]), "=r"(w[8 * i + 3]), "=r"(w[8 * i + 4]), "=r"(w[8 * i + 5]), "=r"(w[8 * i + 6]), "=r"(w[8 * i + 7])
                             : "l"((const uint32_t*)p + 8 * i));
        } else {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) {
                const uint4 a = __ldg((const uint4*)p + i);
                w[4 * i] = a.x; w[4 * i + 1] = a.y; w[4 * i + 2] = a.z; w[4 * i + 3] = a.w;
            }
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0u;
    }
    __device__ __forceinline__ float top() const {
        if constexpr (sizeof(T) == 2) {
            __nv_bfloat162 m = __habs2(pair(0));
#pragma unroll
            for (int i = 1; i < kWords; ++i) m = __hmax2_nan(m, __habs2(pair(i)));
            return max_nan(__low2float(m), __high2float(m));
        } else {
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < kWords; ++i) m = max_nan(m, fabsf(__uint_as_float(w[i])));
            return m;
        }
    }
    __device__ __forceinline__ __nv_bfloat162 pair(int i) const { return *reinterpret_cast<const __nv_bfloat162*>(&w[i]); }
    // Codes of elements 8 q .. 8 q + 7.
    __device__ __forceinline__ uint32_t codes(int q, unsigned long long factor2) const {
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = sizeof(T) == 4 ? w[(8 * q + 2 * i) % kWords] : w[(4 * q + i) % kWords] << 16;
            const uint32_t hi = sizeof(T) == 4 ? w[(8 * q + 2 * i + 1) % kWords] : w[(4 * q + i) % kWords] & 0xffff0000u;
            unsigned long long z;
            asm("mov.b64 %0, {%1, %2};" : "=l"(z) : "r"(lo), "r"(hi));
            asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(z) : "l"(factor2));
            asm("mov.b64 {%0, %1}, %2;" : "=f"(v[2 * i]), "=f"(v[2 * i + 1]) : "l"(z));
        }
        return mx4_e2m1x8(v);
    }
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 5) mx4_quantize_kernel(const T* __restrict__ x, int ld, bool by32, const int32_t* __restrict__ slot_of_row,
                                                                   int k, int64_t x_slots, Mx4View q, int lanes_log2, int chunk) {
    extern __shared__ int32_t smem[];
    grid_dependency_launch();
    grid_dependency_wait();
    const RowMap map(q, smem);
    const int blocks = q.K / 32, ktiles = mx4_ktiles(q.K);
    const Chunks c(q.rows, q.K, lanes_log2, chunk);
    for (int64_t base = c.first; base < c.units; base += c.step) {
        // a lane a unit: its row's place (-1: none) and source (-1: zeros, for a slot that is none), its first block
        int my_row = -1, my_src = -1, my_block = 0;
        if (const int64_t unit = base + (threadIdx.x & 31); (int)(threadIdx.x & 31) < c.chunk && unit < c.units) {
            const int i = c.row_of(unit, my_block);
            my_src = i;
            if (slot_of_row) {
                const int slot = __ldg(slot_of_row + i);
                my_src = slot >= 0 && slot < x_slots ? slot / k : -1;
            }
            my_row = map.at(i);
        }
        for (int r = c.group; r < c.chunk; r += c.per_pass) {
            const int row = __shfl_sync(kAll, my_row, r), src = __shfl_sync(kAll, my_src, r), b = __shfl_sync(kAll, my_block, r) + c.lane;
            const bool mine = row >= 0 && b < blocks;
            Block<T> v;
            if (mine && src >= 0) v.load(x + (int64_t)src * ld + b * 32, by32);
            else v.clear();
            const uint32_t s = mx4_scale_byte(v.top());
            // four blocks' bytes to a word (zero behind the last block of the row)
            uint32_t word = mine ? s << (8 * (b & 3)) : 0u;
            word |= __shfl_xor_sync(kAll, word, 1);
            word |= __shfl_xor_sync(kAll, word, 2);
            if (mine) {
                uint4 codes = make_uint4(0u, 0u, 0u, 0u);
                if (s != 255u) {
                    const unsigned long long factor2 = mx4_factor2(s);
                    codes = make_uint4(v.codes(0, factor2), v.codes(1, factor2), v.codes(2, factor2), v.codes(3, factor2));
                }
                *(uint4*)(q.codes + (int64_t)row * (q.K / 2) + b * 16) = codes;
                if ((b & 3) == 0) *(uint32_t*)(q.scales + mx4_scale_at(row, b, ktiles)) = word;
            }
        }
    }
}

// The eight codes of a word to bf16 numbers, two a register, times the scale (two copies of it): the bytes of the eight magnitudes are looked up four
// codes at a time, the signs put in, and the product with a power of two is exact (an overflow gives infinity).
__device__ __forceinline__ void bf16x8(uint32_t codes, uint32_t scale2, uint32_t* out) {
    // magnitudes 0 0.5 1 1.5 2 3 4 6: bf16 0000 3f00 3f80 3fc0 4000 4040 4080 40c0
    constexpr uint32_t lo0 = 0xc0800000u, lo1 = 0xc0804000u, hi0 = 0x3f3f3f00u, hi1 = 0x40404040u;
    const uint32_t m = codes & 0x77777777u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t sel = m >> (16 * h), sign = codes >> (16 * h);
        const uint32_t lo = __byte_perm(lo0, lo1, sel), hi = __byte_perm(hi0, hi1, sel);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t v = __byte_perm(lo, hi, i == 0 ? 0x5140 : 0x7362);
            v |= ((sign << (12 - 8 * i)) & 0x8000u) | ((sign << (24 - 8 * i)) & 0x80000000u);
            asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(out[2 * h + i]) : "r"(v), "r"(scale2));
        }
    }
}

__device__ __forceinline__ void store32(uint32_t* p, const uint32_t* w) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}

template <typename T>
__global__ void __launch_bounds__(kThreads) mx4_dequantize_kernel(Mx4View q, T* __restrict__ y, int ld, bool by32, int lanes_log2, int chunk) {
    extern __shared__ int32_t smem[];
    grid_dependency_launch();
    grid_dependency_wait();
    const RowMap map(q, smem);
    const int blocks = q.K / 32, ktiles = mx4_ktiles(q.K);
    const Chunks c(q.rows, q.K, lanes_log2, chunk);
    for (int64_t base = c.first; base < c.units; base += c.step) {
        int my_row = -1, my_out = 0, my_block = 0;
        if (const int64_t unit = base + (threadIdx.x & 31); (int)(threadIdx.x & 31) < c.chunk && unit < c.units) {
            my_out = c.row_of(unit, my_block);
            my_row = map.at(my_out);
        }
        for (int r = c.group; r < c.chunk; r += c.per_pass) {
            const int row = __shfl_sync(kAll, my_row, r), i = __shfl_sync(kAll, my_out, r), b = __shfl_sync(kAll, my_block, r) + c.lane;
            if (row < 0 || b >= blocks) continue;
            const uint4 code = __ldg((const uint4*)(q.codes + (int64_t)row * (q.K / 2) + b * 16));
            const uint32_t s = __ldg(q.scales + mx4_scale_at(row, b, ktiles));
            // 2^(s - 127) in bf16: a subnormal for 0, a NaN for 255
            const uint32_t scale = (s == 255u ? 0x7fffu : s ? s << 7 : 0x0040u) * 0x10001u;
            const uint32_t in[4] = {code.x, code.y, code.z, code.w};
            uint32_t* out = (uint32_t*)(y + (int64_t)i * ld + b * 32);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t w[8];
                bf16x8(in[j], scale, w);
                if constexpr (sizeof(T) == 2) {
                    if (by32) {
                        if (j & 1) continue;                           // the two codes of a 32-byte store together
                        bf16x8(in[j + 1], scale, w + 4);
                        store32(out + 4 * j, w);
                    } else {
                        *(uint4*)(out + 4 * j) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                } else {
                    const uint32_t f[8] = {w[0] << 16, w[0] & 0xffff0000u, w[1] << 16, w[1] & 0xffff0000u, w[2] << 16, w[2] & 0xffff0000u, w[3] << 16, w[3] & 0xffff0000u};
                    if (by32) {
                        store32(out + 8 * j, f);
                    } else {
                        *(uint4*)(out + 8 * j) = make_uint4(f[0], f[1], f[2], f[3]);
                        *(uint4*)(out + 8 * j + 4) = make_uint4(f[4], f[5], f[6], f[7]);
                    }
                }
            }
        }
    }
}

int lanes_log2_of(int K) {
    int l = 2;                         // four lanes put a word of scale bytes together
    while (l < 5 && (1 << l) < K / 32) ++l;
    return l;
}
// Units a warp looks up at once: as many as leave every SM's 48 warps the same number of chunks (nine tenths of it at least).  Grouped rows,
// whose look-up costs as much as their codes: 32, if that leaves 16 warps an SM (131072 rows of 256: 20 us with four, 15 with 32).
struct Shape {
    int lanes_log2, chunk, grid;
    Shape(int64_t rows, int K, bool grouped) {
        lanes_log2 = lanes_log2_of(K);
        const int64_t warps = (int64_t)gemm_tc_sm_count() * 48, units = rows * ((K + 1023) / 1024);
        const int per_pass = 32 >> lanes_log2;
        int64_t trips;
        for (chunk = 32;; chunk /= 2) {
            const int64_t chunks = (units + chunk - 1) / chunk;
            trips = (chunks + warps - 1) / warps;
            const int64_t used = (chunks + trips - 1) / trips;         // warps, all with the same number of trips
            grid = (int)((used + kThreads / 32 - 1) / (kThreads / 32));
            if (chunk == per_pass || (grouped ? 3 * chunks >= warps : 10 * chunks >= 9 * trips * warps)) break;
        }
    }
};
// Do rows allow 32-byte accesses?
bool rows_by_32(const void* p, int dtype, int64_t ld) { return (uintptr_t)p % 32 == 0 && ld * (dtype == BIGMAC_BF16 ? 2 : 4) % 32 == 0; }
size_t map_bytes(const Mx4View& q) { return q.offsets ? (size_t)(2 * q.E + 2) * 4 : 0; }

}  // namespace

cudaError_t launch_mx4_quantize(const void* x, int dtype, int64_t ld, const int32_t* slot_of_row, int k, int x_rows, const Mx4View& q,
                                cudaStream_t stream) {
    if (q.rows == 0) return cudaSuccess;
    const Shape z(q.rows, q.K, q.offsets != nullptr);
    const int64_t slots = (int64_t)x_rows * k;
    const bool by32 = rows_by_32(x, dtype, ld);
    if (dtype == BIGMAC_BF16)
        return launch_chained(mx4_quantize_kernel<__nv_bfloat16>, z.grid, kThreads, map_bytes(q), stream, (const __nv_bfloat16*)x, (int)ld, by32, slot_of_row, k,
                              slots, q, z.lanes_log2, z.chunk);
    return launch_chained(mx4_quantize_kernel<float>, z.grid, kThreads, map_bytes(q), stream, (const float*)x, (int)ld, by32, slot_of_row, k, slots, q, z.lanes_log2, z.chunk);
}

cudaError_t launch_mx4_dequantize(const Mx4View& q, void* y, int dtype, int64_t ld, cudaStream_t stream) {
    if (q.rows == 0) return cudaSuccess;
    const Shape z(q.rows, q.K, q.offsets != nullptr);
    const bool by32 = rows_by_32(y, dtype, ld);
    if (dtype == BIGMAC_BF16)
        return launch_chained(mx4_dequantize_kernel<__nv_bfloat16>, z.grid, kThreads, map_bytes(q), stream, q, (__nv_bfloat16*)y, (int)ld, by32, z.lanes_log2, z.chunk);
    return launch_chained(mx4_dequantize_kernel<float>, z.grid, kThreads, map_bytes(q), stream, q, (float*)y, (int)ld, by32, z.lanes_log2, z.chunk);
}

}  // namespace bigmac
