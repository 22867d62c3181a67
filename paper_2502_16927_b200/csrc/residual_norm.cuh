// Pieces that the forward and the backward kernels of the joint share: a row on its threads, its sums, its inputs on their way
// through shared memory.
#pragma once
#include "residual_norm.h"

namespace bigmac {
namespace resnorm {

constexpr unsigned kAll = 0xffffffffu;

// Row `row` of a matrix.
template <typename T>
__device__ __forceinline__ T* row_at(T* p, int row, int ld) { return p + (int64_t)row * ld; }

struct Params {
    const void *x, *y, *gate, *dr, *dn;
    void *r, *n, *dx, *dy, *dgate;
    int x_ld, y_ld, gate_ld, dr_ld, dn_ld, r_ld, n_ld, dx_ld, dy_ld, dgate_ld;      // 32 bits: a row's place is one wide multiplication
    const float *w_post, *b_post, *w_pre, *b_pre;
    float4* stats;
    float* partial;
    float rho, post_eps, pre_eps, inv_d;
    int T, d, post, pre, gate_kind;
};

// Two fp32 numbers in a register pair: one instruction for two elements (sm_100 f32x2 arithmetic).
typedef unsigned long long f2;
__device__ __forceinline__ f2 pk(float a, float b) { f2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ f2 pk(float a) { return pk(a, a); }
__device__ __forceinline__ void upk(f2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ float both(f2 v) { float a, b; upk(v, a, b); return a + b; }
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) { f2 d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c)); return d; }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) { f2 d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ f2 add2(f2 a, f2 b) { f2 d; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }

// A row's elements on its threads: thread t has pieces v of eight.  VEC kNeighbours: eight neighbours (a 16-byte access of bf16); kFours: four and
// four, each a 16-byte access of fp32 next to the other threads' (eight neighbours are two accesses that use half of every 32-byte sector: backward of 8000 rows of
// 4096 292 us, in fours 187).  kAlternate, for rows off 16-byte boundaries: the elements of a warp's threads alternate, so that accesses to single
// elements are still whole lines, at constant distances (8000 rows of 1357 with the elements of a row's threads alternating 44 us and 79 for the backward, so 34 and 70).
constexpr int kAlternate = 0, kNeighbours = 1, kFours = 2;
template <typename T>
constexpr int kVecOf = sizeof(T) == 4 ? kFours : kNeighbours;
template <int VEC>
__device__ __forceinline__ int column(int v, int j, int t, int threads) {
    return VEC == kNeighbours ? (v * threads + t) * 8 + j : VEC == kFours ? (2 * v + (j >> 2)) * 4 * threads + 4 * t + (j & 3) : (v * threads + (t & ~31)) * 8 + 32 * j + (t & 31);
}

__device__ __forceinline__ f2 pair_of(uint32_t w) { return pk(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ void unpack8(const uint4& a, f2* f) { f[0] = pair_of(a.x); f[1] = pair_of(a.y); f[2] = pair_of(a.z); f[3] = pair_of(a.w); }
__device__ __forceinline__ void fill8(float v, f2* f) { f[0] = f[1] = f[2] = f[3] = pk(v); }
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_float(float v, float* p) { *p = v; }
__device__ __forceinline__ void from_float(float v, __nv_bfloat16* p) { *p = __float2bfloat16(v); }

// Eight elements of a row (zeros behind column d).
template <typename T, int VEC>
__device__ __forceinline__ void load8(const T* row, int v, int t, int threads, int d, f2* f) {
    const int c0 = column<VEC>(v, 0, t, threads);
    if constexpr (VEC == kFours) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = column<VEC>(v, 4 * h, t, threads);
            const ulonglong2 a = c < d ? *(const ulonglong2*)(row + c) : make_ulonglong2(0, 0);
            f[2 * h] = a.x; f[2 * h + 1] = a.y;
        }
    } else if constexpr (VEC) {
        if (c0 < d) {
            if constexpr (sizeof(T) == 2) {
                unpack8(*(const uint4*)(row + c0), f);
            } else {
                const ulonglong2 a = *(const ulonglong2*)(row + c0), b = *(const ulonglong2*)(row + c0 + 4);
                f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
            }
        } else {
            fill8(0.0f, f);
        }
    } else {
        float e[8];
        if (c0 + 7 * 32 < d) {
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = to_float(row[c0 + j * 32]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = c0 + j * 32 < d ? to_float(row[c0 + j * 32]) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = pk(e[2 * j], e[2 * j + 1]);
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void store8(T* row, int v, int t, int threads, int d, const f2* f) {
    const int c0 = column<VEC>(v, 0, t, threads);
    float e[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) upk(f[j], e[2 * j], e[2 * j + 1]);
    if constexpr (VEC == kFours) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (const int c = column<VEC>(v, 4 * h, t, threads); c < d) *(ulonglong2*)(row + c) = make_ulonglong2(f[2 * h], f[2 * h + 1]);
    } else if constexpr (VEC) {
        if (c0 >= d) return;
        if constexpr (sizeof(T) == 2) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(e[2 * i], e[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&b);
            }
            *(uint4*)(row + c0) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            *(float4*)(row + c0) = make_float4(e[0], e[1], e[2], e[3]);
            *(float4*)(row + c0 + 4) = make_float4(e[4], e[5], e[6], e[7]);
        }
    } else {
        if (c0 + 7 * 32 < d) {
#pragma unroll
            for (int j = 0; j < 8; ++j) from_float(e[j], row + c0 + j * 32);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c0 + j * 32 < d) from_float(e[j], row + c0 + j * 32);
        }
    }
}
// Zeros behind column d.
template <int VEC>
__device__ __forceinline__ void cut8(int v, int t, int threads, int d, f2* f) {
    const int c0 = column<VEC>(v, 0, t, threads);
    if constexpr (VEC == kFours) {
        if (c0 >= d) f[0] = f[1] = pk(0.0f);
        if (column<VEC>(v, 4, t, threads) >= d) f[2] = f[3] = pk(0.0f);
    } else if constexpr (VEC) {
        if (c0 >= d) fill8(0.0f, f);
    } else if (c0 + 7 * 32 >= d) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float a, b;
            upk(f[j], a, b);
            f[j] = pk(c0 + 64 * j < d ? a : 0.0f, c0 + 64 * j + 32 < d ? b : 0.0f);
        }
    }
}
// A vector of parameters: `fill` where there is none.  (The pointers of VEC vectors are 16-byte aligned, too.)
template <int VEC>
__device__ __forceinline__ void param8(const float* p, float fill, int v, int t, int threads, int d, f2* f) {
    if (p) load8<float, VEC>(p, v, t, threads, d, f);
    else fill8(fill, f);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
    return v;
}
// Two sums for little more than one: after the first step the lower half of the warp goes on with a, the upper one with b (which
// then hold the sums).
__device__ __forceinline__ float warp_sum_halves(float a, float b, bool upper) {
    float v = upper ? b : a;
    v += __shfl_xor_sync(kAll, upper ? a : b, 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
    return v;
}
// Waits for the `threads` threads of a row (whole warps of one block; id 1 .. 15).
__device__ __forceinline__ void row_barrier(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// What a row's threads have in common: their number, and room for sums, two regions in turn, so that one barrier a sum is enough.  A region holds
// the warps' (16 at most) parts of two sums, zeros behind them.
struct Row {
    float *slots, *other;
    int t, threads, id;
    __device__ __forceinline__ Row(float* a, float* b, int t_, int threads_, int id_) : slots(a), other(b), t(t_), threads(threads_), id(id_) {
        if (t < 16 && t >= threads >> 5) a[t] = a[16 + t] = b[t] = b[16 + t] = 0.0f;       // seen behind the first sum's barrier
    }
    __device__ __forceinline__ void turn() { float* const s = slots; slots = other; other = s; }
};
// The warps' parts, read by every thread: half the latency of adding them up between lanes.
__device__ __forceinline__ float slots_sum(const float* slots, int threads) {
    const ulonglong2* q = (const ulonglong2*)slots;
    f2 s = add2(q[0].x, q[0].y);
    if (threads > 128) s = add2(s, add2(q[1].x, q[1].y));
    if (threads > 256) s = add2(s, add2(add2(q[2].x, q[2].y), add2(q[3].x, q[3].y)));
    return both(s);
}
// Sums over the threads of a row, in a fixed order.
__device__ __forceinline__ float row_sum(float v, Row& r) {
    v = warp_sum(v);
    if (r.threads == 32) return v;
    if ((r.t & 31) == 0) r.slots[r.t >> 5] = v;
    row_barrier(r.id, r.threads);
    v = slots_sum(r.slots, r.threads);
    r.turn();
    return v;
}
// Two at once.
__device__ __forceinline__ void row_sum2(float& a, float& b, Row& r) {
    const int lane = r.t & 31;
    float v = warp_sum_halves(a, b, lane >= 16);
    if (r.threads > 32) {
        if ((lane & 15) == 0) r.slots[(lane & 16) + (r.t >> 5)] = v;
        row_barrier(r.id, r.threads);
        v = slots_sum(r.slots + (lane & 16), r.threads);
        r.turn();
    }
    a = __shfl_sync(kAll, v, 0);
    b = __shfl_sync(kAll, v, 16);
}

// Mean and 1 / sqrt(var + eps) of a row in registers (zeros behind column d); the variance from the differences to the mean.
template <int NV, int VEC>
__device__ __forceinline__ void row_stats(int kind, const f2* f, float eps, const Params& p, Row& row, float& mean, float& rstd) {
    mean = 0.0f;
    rstd = 1.0f;
    if (kind == BIGMAC_NORM_NONE) return;
    f2 s = pk(0.0f);
    if (kind == BIGMAC_NORM_LAYER) {
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) s = add2(s, f[i]);
        // the quotient, rounded once (a step of Newton's on the product with 1 / d): a row of equal elements has that element as its mean and a norm of
        // zeros, where the product alone, a unit of 2^-23 off, left as much divided by sqrt(eps) (5152 everywhere, 1000 columns: 0.4)
        const float sum = row_sum(both(s), row);
        mean = sum * p.inv_d;
        mean = fmaf(fmaf(-mean, (float)p.d, sum), p.inv_d, mean);
        s = pk(0.0f);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            f2 e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) e[j] = add2(f[4 * v + j], pk(-mean));
            if (!VEC) cut8<VEC>(v, row.t, row.threads, p.d, e);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (VEC && column<VEC>(v, VEC == kFours ? 4 * h : 0, row.t, row.threads) >= p.d) continue;
                s = fma2(e[2 * h], e[2 * h], s);
                s = fma2(e[2 * h + 1], e[2 * h + 1], s);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) s = fma2(f[i], f[i], s);
    }
    rstd = rsqrtf(fmaf(row_sum(both(s), row), p.inv_d, eps));          // within two units of 2^-24
}


// ---- persistent blocks: rows on their way through shared memory, parameters in it

constexpr int kThreads = 512;
constexpr int kNoBlock = -1, kAnyGate = -2;                            // GATE: no y; by p.y and p.gate_kind
constexpr uint32_t kPieceBytes = kThreads * 16;                        // a 16-byte piece of every thread

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void wait_groups(int pending) {
    switch (pending) {
        case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
        case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
        case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
        default: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
    }
}

// Bytes of one tensor's row in a stage where rows lie at any address: the 16-byte granules that it touches.
__host__ __device__ inline uint32_t granule_bytes(int d, int es) { return (uint32_t)(d * es / 16 + 2) * 16; }
// Bytes of a stage of a block whose rows have `count` tensors.
inline size_t stage_bytes(bool vec, int d, int es, int groups, int count, int nv = 1) {
    return vec ? (size_t)count * nv * (es / 2) * kPieceBytes : (size_t)count * groups * granule_bytes(d, es);
}

// The rows a group of threads works on, `stages` of them in shared memory or on their way there.
// VEC: every thread copies and reads its own 16 bytes, so no thread waits for another.  Else a row begins anywhere: its threads copy the 16-byte
// granules that hold it and read single elements after a barrier; the first and the last rows of all, whose granules may reach out of the
// tensor, are read directly.
template <typename T, int VEC, int COUNT, int NV = 1>
struct Ring {
    static constexpr int kHalves = (int)sizeof(T) / 2;                 // 16-byte pieces of eight elements
    const T* in[COUNT];
    int ld[COUNT];
    bool has[COUNT];
    uint8_t* base;                                                     // VEC: the thread's first slot; else the group's
    int stages, T_rows, d;
    uint32_t granules;                                                 // !VEC: bytes of a tensor's row

    __device__ __forceinline__ void init(uint8_t* smem, int group, int stages_, const Params& p) {
        stages = stages_; T_rows = p.T; d = p.d;
        granules = granule_bytes(p.d, (int)sizeof(T));
        base = VEC ? smem + threadIdx.x * 16 : smem + (size_t)group * stages * COUNT * granules;
    }
    __device__ __forceinline__ uint8_t* slot(int stage, int which) const {
        return base + (VEC ? (uint32_t)(stage * COUNT + which) * NV * kHalves * kPieceBytes : (uint32_t)(stage * COUNT + which) * granules);
    }
    // Fewer than 16 bytes of the tensor before or behind the row.
    __device__ __forceinline__ bool direct(int row) const { return !VEC && ((int64_t)row * d < 16 || (int64_t)(T_rows - 1 - row) * d < 16); }
    __device__ __forceinline__ void fetch(int stage, int row, int t, int threads) {
        if (row < T_rows && !direct(row)) {
            if constexpr (VEC) {
#pragma unroll
                for (int i = 0; i < COUNT; ++i) {
                    if (!has[i]) continue;
                    const T* from = row_at(in[i], row, ld[i]);
                    const uint32_t to = (uint32_t)__cvta_generic_to_shared(slot(stage, i));
#pragma unroll
                    for (int v = 0; v < NV; ++v) {
#pragma unroll
                        for (int h = 0; h < kHalves; ++h)
                            if (const int c = column<VEC>(v, 4 * h, t, threads); c < d) copy16(to + (v * kHalves + h) * kPieceBytes, from + c);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < COUNT; ++i) {
                    if (!has[i]) continue;
                    const uintptr_t from = (uintptr_t)row_at(in[i], row, ld[i]);
                    const uint8_t* first = (const uint8_t*)(from & ~(uintptr_t)15);
                    const uint32_t bytes = (uint32_t)(from & 15) + d * (uint32_t)sizeof(T);
                    const uint32_t to = (uint32_t)__cvta_generic_to_shared(slot(stage, i));
                    for (uint32_t at = t * 16; at < bytes; at += threads * 16) copy16(to + at, first + at);
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // The first rows are asked for; LATE: as many as there are stages, which `again` then fills.
    template <bool LATE = false>
    __device__ __forceinline__ void start(int first, int step, int t, int threads) {
        for (int s = 0; s < stages - (LATE ? 0 : 1); ++s) fetch(s, first + s * step, t, threads);
    }
    // LATE (VEC): row `row` is in its stage; once it has been read, the row that is `stages` rows later comes there.
    __device__ __forceinline__ void arrived() const { wait_groups(stages - 1); }
    __device__ __forceinline__ void again(int stage, int row, int step, const Row& at) { fetch(stage, row + stages * step, at.t, at.threads); }
    // Row `row` is in its stage, the one stages - 1 rows later on its way.
    __device__ __forceinline__ void next(int stage, int row, int step, const Row& at) {
        if constexpr (VEC) {
            fetch(stage == 0 ? stages - 1 : stage - 1, row + (stages - 1) * step, at.t, at.threads);
            wait_groups(stages - 1);
        } else {
            if (stages > 1) wait_groups(stages - 2);
            sync(at);                                                  // the row before has been read by all, this one written
            fetch(stage == 0 ? stages - 1 : stage - 1, row + (stages - 1) * step, at.t, at.threads);
            if (stages == 1) {
                wait_groups(0);
                sync(at);
            }
        }
    }
    static __device__ __forceinline__ void sync(const Row& at) {
        if (at.threads == 32) __syncwarp();
        else row_barrier(at.id, at.threads);
    }
    // Piece v of a row.
    __device__ __forceinline__ void get(int stage, int which, int v, int row, int t, int threads, f2* f) const {
        if (!has[which]) { fill8(0.0f, f); return; }
        if constexpr (VEC) {
            const uint8_t* s = slot(stage, which) + v * kHalves * kPieceBytes;
            if constexpr (sizeof(T) == 2) {
                if (column<VEC>(v, 0, t, threads) < d) unpack8(*(const uint4*)s, f);
                else fill8(0.0f, f);
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const ulonglong2 a = column<VEC>(v, 4 * h, t, threads) < d ? *(const ulonglong2*)(s + h * kPieceBytes) : make_ulonglong2(0, 0);
                    f[2 * h] = a.x; f[2 * h + 1] = a.y;
                }
            }
        } else {
            const T* from = row_at(in[which], row, ld[which]);
            // (two loads: through one pointer to either, every element costs a 64-bit address)
            if (direct(row)) load8<T, kAlternate>(from, v, t, threads, d, f);
            else load8<T, kAlternate>((const T*)(slot(stage, which) + ((uintptr_t)from & 15)), v, t, threads, d, f);
        }
    }
};

// Vectors of parameters in shared memory: piece v of vector `which`, 32 bytes in two pieces.  Every thread its own columns, which takes constant
// offsets (7 % of the forward with eight columns a thread); SHARED: the rows of a block read one copy, where there is no room for that.
template <int NV, bool SHARED>
struct ParamStore {
    uint8_t* base;                                                     // the thread's first piece
    uint32_t row_step;                                                 // SHARED: from piece to piece, 16 bytes of every thread of a row
    __device__ __forceinline__ ParamStore(uint8_t* smem, int t, int threads) : base(smem + (SHARED ? t : (int)threadIdx.x) * 16), row_step(threads * 16) {}
    __device__ __forceinline__ uint32_t step() const { return SHARED ? row_step : kPieceBytes; }
    __device__ __forceinline__ uint8_t* at(int which, int v) const { return base + (uint32_t)(2 * (which * NV + v)) * step(); }
    __device__ __forceinline__ void put(int which, int v, const f2* f) {
        *(ulonglong2*)at(which, v) = make_ulonglong2(f[0], f[1]);
        *(ulonglong2*)(at(which, v) + step()) = make_ulonglong2(f[2], f[3]);
    }
    __device__ __forceinline__ void get(int which, int v, f2* f) const {
        const ulonglong2 a = *(const ulonglong2*)at(which, v), b = *(const ulonglong2*)(at(which, v) + step());
        f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
    }
};
// Bytes of one vector.
__host__ __device__ inline uint32_t param_bytes(bool shared, int threads, int nv) { return (uint32_t)(shared ? threads : kThreads) * nv * 32; }
// w_post and b_post, a channel gate multiplied in (gate (hat w + b) = hat (gate w) + gate b); zeros behind column d, so that what they multiply adds
// nothing to a sum there.
template <int VEC>
__device__ __forceinline__ void post_params(const Params& p, int v, int t, int threads, f2* w, f2* b) {
    param8<VEC>(p.w_post, 1.0f, v, t, threads, p.d, w);
    param8<VEC>(p.b_post, 0.0f, v, t, threads, p.d, b);
    if (p.gate_kind == BIGMAC_GATE_CHANNEL) {
        f2 g[4];
        load8<float, VEC>((const float*)p.gate, v, t, threads, p.d, g);
#pragma unroll
        for (int j = 0; j < 4; ++j) { w[j] = mul2(w[j], g[j]); b[j] = mul2(b[j], g[j]); }
    }
    cut8<VEC>(v, t, threads, p.d, w);
    cut8<VEC>(v, t, threads, p.d, b);
}

Params params_of(const ResNorm& a);
// Threads of a row of d columns, 8 nv of them each: whole warps, kThreads at most.
static_assert(kResNormMaxWidth <= 16 * kThreads, "16 columns a thread at most: a row's warps have 16 places for their sums");
inline int threads_of(int d, int nv) { return (d + 8 * nv * 32 - 1) / (8 * nv * 32) * 32; }

}  // namespace resnorm
}  // namespace bigmac
