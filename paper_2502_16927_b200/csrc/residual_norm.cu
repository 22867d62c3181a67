// The joint of two blocks of a network, forward and backward:
//
//     hat = (y - mu) s              a = hat * w_post + b_post                s = 1 / sqrt(var + eps)     (RMS norm: mu = 0, var = mean y^2)
//     r   = rho x + gate * a        n = ((r - mu_r) s_r) * w_pre + b_pre
//
//     q   = dn * w_pre              D  = dr + s_r (q - mean(q) - hat_r mean(q hat_r))                  (RMS: without mean(q))
//     dx  = rho D                   p  = gate D w_post                       dy = s (p - mean(p) - hat mean(p hat))
//     dw_post = sum gate D hat      db_post = sum gate D                     dgate = D a, summed over what the gate is shared by
//     dw_pre  = sum dn hat_r        db_pre  = sum dn                         (sums over the rows)
//
// All in fp32; r goes into its norm as it is before it is rounded to the output's type, and the backward pass computes it again from x and y (no
// more bytes than reading r, and exact).  Bound by memory: forward x, y (and a full gate) in, r, n out; backward x, y, dr, dn in,
// dx, dy out.  Both read every tensor once: a row lies in the registers of one to 32 warps, which share its sums.
#include "residual_norm.h"

namespace bigmac {

namespace {

constexpr unsigned kAll = 0xffffffffu;

struct Params {
    const void *x, *y, *gate, *dr, *dn;
    void *r, *n, *dx, *dy, *dgate;
    int64_t x_ld, y_ld, gate_ld, dr_ld, dn_ld, r_ld, n_ld, dx_ld, dy_ld, dgate_ld;
    const float *w_post, *b_post, *w_pre, *b_pre;
    float4* stats;
    float* partial;
    float rho, post_eps, pre_eps, inv_d;
    int T, d, post, pre, gate_kind;
};

// Element j of thread t's piece v.  VEC: eight neighbours a thread, 16-byte loads.  Else the threads' elements alternate, so that
// loads of single elements are still whole lines.
template <bool VEC>
__device__ __forceinline__ int column(int v, int j, int t, int threads) { return VEC ? (v * threads + t) * 8 + j : (v * 8 + j) * threads + t; }

__device__ __forceinline__ void unpack8(const uint4& a, float* f) {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_float(float v, float* p) { *p = v; }
__device__ __forceinline__ void from_float(float v, __nv_bfloat16* p) { *p = __float2bfloat16(v); }

// Eight elements of a row (zeros behind column d).
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int v, int t, int threads, int d, float* f) {
    const int c0 = column<VEC>(v, 0, t, threads);
    if constexpr (VEC) {
        if (c0 < d) {
            if constexpr (sizeof(T) == 2) {
                unpack8(*(const uint4*)(row + c0), f);
            } else {
                const float4 a = *(const float4*)(row + c0), b = *(const float4*)(row + c0 + 4);
                f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = 0.0f;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = c0 + j * threads;
            f[j] = c < d ? to_float(row[c]) : 0.0f;
        }
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* row, int v, int t, int threads, int d, const float* f) {
    const int c0 = column<VEC>(v, 0, t, threads);
    if constexpr (VEC) {
        if (c0 >= d) return;
        if constexpr (sizeof(T) == 2) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&b);
            }
            *(uint4*)(row + c0) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            *(float4*)(row + c0) = make_float4(f[0], f[1], f[2], f[3]);
            *(float4*)(row + c0 + 4) = make_float4(f[4], f[5], f[6], f[7]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = c0 + j * threads;
            if (c < d) from_float(f[j], row + c);
        }
    }
}
// A vector of parameters: fill where there is none.  (The pointers of VEC vectors are 16-byte aligned, too.)
template <bool VEC>
__device__ __forceinline__ void param8(const float* p, float fill, int v, int t, int threads, int d, float* f) {
    if (p) {
        load8<float, VEC>(p, v, t, threads, d, f);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = fill;
    }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
    return v;
}
// Waits for the `threads` threads of a row (whole warps of one block; id 1 .. 15).
__device__ __forceinline__ void row_barrier(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// Sums of N values over the threads of a row, in a fixed order.  `slots`: N x 32 floats of shared memory of the row, alternating
// between two such regions from sum to sum, so that one barrier each is enough.
template <int N>
__device__ __forceinline__ void row_sum(float* s, float* slots, int t, int threads, int id) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = warp_sum(s[i]);
    if (threads == 32) return;
    const int lane = t & 31, warp = t >> 5, warps = threads >> 5;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) slots[i * 32 + warp] = s[i];
    }
    row_barrier(id, threads);
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = warp_sum(lane < warps ? slots[i * 32 + lane] : 0.0f);
}

// Mean and 1 / sqrt(var + eps) of a row in registers; the variance from the differences to the mean.
template <int NV, bool VEC>
__device__ __forceinline__ void row_stats(int kind, const float* f, float eps, float inv_d, int d, int t, int threads, float*& slots, float*& other,
                                          int id, float& mean, float& rstd) {
    mean = 0.0f;
    rstd = 1.0f;
    if (kind == BIGMAC_NORM_NONE) return;
    float s[1];
    if (kind == BIGMAC_NORM_LAYER) {
        s[0] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8 * NV; ++i) s[0] += f[i];
        row_sum<1>(s, slots, t, threads, id);
        float* const swap = slots; slots = other; other = swap;
        mean = s[0] * inv_d;
    }
    s[0] = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float e = column<VEC>(v, j, t, threads) < d ? f[8 * v + j] - mean : 0.0f;
            s[0] = fmaf(e, e, s[0]);
        }
    row_sum<1>(s, slots, t, threads, id);
    float* const swap = slots; slots = other; other = swap;
    rstd = 1.0f / sqrtf(fmaf(s[0], inv_d, eps));
}

// One row to `threads` threads (a block holds blockDim.x / threads rows).
template <typename T, int NV, bool VEC>
__global__ void __launch_bounds__(1024 / NV) residual_norm_kernel(const Params p, int threads) {
    __shared__ float sums[2][32 * 8];
    grid_dependency_launch();
    grid_dependency_wait();
    const int t = threadIdx.x % threads, in_block = threadIdx.x / threads, id = 1 + in_block;
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x / threads) + in_block;
    if (row >= p.T) return;                                            // whole rows of threads
    float *slots = sums[0], *other = sums[1];                          // rows of more than a warp have a block for themselves
    float r[8 * NV], y[8 * NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) load8<T, VEC>((const T*)p.x + row * p.x_ld, v, t, threads, p.d, r + 8 * v);
    float4 st = make_float4(0.0f, 1.0f, 0.0f, 1.0f);
    if (p.y) {
#pragma unroll
        for (int v = 0; v < NV; ++v) load8<T, VEC>((const T*)p.y + row * p.y_ld, v, t, threads, p.d, y + 8 * v);
        const float token_gate = p.gate_kind == BIGMAC_GATE_TOKEN ? ((const float*)p.gate)[row] : 1.0f;
        row_stats<NV, VEC>(p.post, y, p.post_eps, p.inv_d, p.d, t, threads, slots, other, id, st.x, st.y);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float w[8], b[8], g[8];
            param8<VEC>(p.w_post, 1.0f, v, t, threads, p.d, w);
            param8<VEC>(p.b_post, 0.0f, v, t, threads, p.d, b);
            if (p.gate_kind == BIGMAC_GATE_FULL) {
                load8<T, VEC>((const T*)p.gate + row * p.gate_ld, v, t, threads, p.d, g);
            } else if (p.gate_kind == BIGMAC_GATE_CHANNEL) {
                load8<float, VEC>((const float*)p.gate, v, t, threads, p.d, g);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] = token_gate;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float a = fmaf((y[8 * v + j] - st.x) * st.y, w[j], b[j]);
                r[8 * v + j] = column<VEC>(v, j, t, threads) < p.d ? fmaf(p.rho, r[8 * v + j], g[j] * a) : 0.0f;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8 * NV; ++i) r[i] *= p.rho;
    }
    if (p.r) {
#pragma unroll
        for (int v = 0; v < NV; ++v) store8<T, VEC>((T*)p.r + row * p.r_ld, v, t, threads, p.d, r + 8 * v);
    }
    if (p.n) {
        row_stats<NV, VEC>(p.pre, r, p.pre_eps, p.inv_d, p.d, t, threads, slots, other, id, st.z, st.w);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float w[8], b[8];
            param8<VEC>(p.w_pre, 1.0f, v, t, threads, p.d, w);
            param8<VEC>(p.b_pre, 0.0f, v, t, threads, p.d, b);
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = fmaf((r[8 * v + j] - st.z) * st.w, w[j], b[j]);
            store8<T, VEC>((T*)p.n + row * p.n_ld, v, t, threads, p.d, w);
        }
    }
    if (p.stats && t == 0) p.stats[row] = st;
}

// ------------------------------------------------------------------------------------------ backward

constexpr int kBwdThreads = 512;
enum { IN_X = 0, IN_Y, IN_DR, IN_DN, IN_GATE, IN_COUNT };

__device__ __forceinline__ void copy16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}

// Persistent blocks of 512 threads, `threads` of them to a row, 8 NV columns a thread; a thread keeps the column sums of its
// columns over its rows.  VEC: the inputs of the next STAGES - 1 rows are on their way to shared memory while a row is worked on
// (every thread copies and reads its own 16 bytes: no barrier); 40 KB a stage and SM in bf16.
template <typename T, int NV, bool VEC, int STAGES>
__global__ void __launch_bounds__(kBwdThreads, 1) residual_norm_bwd_kernel(const Params p, int threads) {
    extern __shared__ __align__(16) uint8_t ring[];
    constexpr int kPieces = NV * (int)sizeof(T) / 2;                   // 16-byte pieces of a row a thread has
    __shared__ float sums[2][kBwdThreads / 32][4 * 32];
    grid_dependency_launch();
    grid_dependency_wait();
    const int t = threadIdx.x % threads, group = threadIdx.x / threads, groups = kBwdThreads / threads, id = 1 + group;
    const int64_t first = (int64_t)blockIdx.x * groups + group, step = (int64_t)gridDim.x * groups;
    const bool working = group < groups;                               // threads that are no whole row rest
    float *slots = sums[0][working ? group : 0], *other = sums[1][working ? group : 0];

    const T* in[IN_COUNT] = {(const T*)p.x, (const T*)p.y, (const T*)p.dr, (const T*)p.dn, p.gate_kind == BIGMAC_GATE_FULL ? (const T*)p.gate : nullptr};
    const int64_t ld[IN_COUNT] = {p.x_ld, p.y_ld, p.dr_ld, p.dn_ld, p.gate_ld};
    auto slot_of = [&](int stage, int which, int piece) { return ring + ((size_t)((stage * IN_COUNT + which) * kPieces + piece) * kBwdThreads + threadIdx.x) * 16; };
    auto fetch = [&](int stage, int64_t row) {
        if (row < p.T) {
#pragma unroll
            for (int i = 0; i < IN_COUNT; ++i) {
                if (!in[i]) continue;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const int c = column<true>(v, 0, t, threads);
                    if (c >= p.d) continue;
#pragma unroll
                    for (int h = 0; h < (int)sizeof(T) / 2; ++h) copy16(slot_of(stage, i, v * (int)sizeof(T) / 2 + h), in[i] + row * ld[i] + c + h * 4);
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto get = [&](int stage, int which, int v, int64_t row, float* f) {
        if (!in[which]) {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = 0.0f;
        } else if constexpr (VEC) {
            if (column<true>(v, 0, t, threads) < p.d) {
                if constexpr (sizeof(T) == 2) {
                    unpack8(*(const uint4*)slot_of(stage, which, v), f);
                } else {
                    const float4 a = *(const float4*)slot_of(stage, which, 2 * v), b = *(const float4*)slot_of(stage, which, 2 * v + 1);
                    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = 0.0f;
            }
        } else {
            load8<T, false>(in[which] + row * ld[which], v, t, threads, p.d, f);
        }
    };

    float sum_post_w[8 * NV], sum_post_b[8 * NV], sum_pre_w[8 * NV], sum_pre_b[8 * NV];
#pragma unroll
    for (int i = 0; i < 8 * NV; ++i) sum_post_w[i] = sum_post_b[i] = sum_pre_w[i] = sum_pre_b[i] = 0.0f;

    if (working) {
        if (VEC) {
#pragma unroll
            for (int s = 0; s < STAGES - 1; ++s) fetch(s, first + s * step);
        }
        int stage = 0;
        float4 next_stats = first < p.T ? p.stats[first] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int64_t row = first; row < p.T; row += step, stage = stage + 1 == STAGES ? 0 : stage + 1) {
            const float4 st = next_stats;
            if (row + step < p.T) next_stats = p.stats[row + step];
            const float token_gate = p.gate_kind == BIGMAC_GATE_TOKEN ? ((const float*)p.gate)[row] : 1.0f;
            if (VEC) {
                fetch(stage + STAGES - 1 >= STAGES ? stage - 1 : stage + STAGES - 1, row + (STAGES - 1) * step);
                asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
            }
            float hat[8 * NV], a[8 * NV], g[8 * NV], D[8 * NV];
            {
                // r, its norm's gradient: q = dn w_pre, sums of q and q hat_r
                float hat_r[8 * NV], q[8 * NV], s[2] = {0.0f, 0.0f};
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float w[8], b[8], in8[8];
                    get(stage, IN_X, v, row, in8);
#pragma unroll
                    for (int j = 0; j < 8; ++j) hat_r[8 * v + j] = p.rho * in8[j];
                    if (p.y) {
                        get(stage, IN_Y, v, row, in8);
                        param8<VEC>(p.w_post, 1.0f, v, t, threads, p.d, w);
                        param8<VEC>(p.b_post, 0.0f, v, t, threads, p.d, b);
                        if (p.gate_kind == BIGMAC_GATE_FULL) {
                            get(stage, IN_GATE, v, row, g + 8 * v);
                        } else if (p.gate_kind == BIGMAC_GATE_CHANNEL) {
                            load8<float, VEC>((const float*)p.gate, v, t, threads, p.d, g + 8 * v);
                        } else {
#pragma unroll
                            for (int j = 0; j < 8; ++j) g[8 * v + j] = token_gate;
                        }
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            hat[8 * v + j] = (in8[j] - st.x) * st.y;
                            a[8 * v + j] = fmaf(hat[8 * v + j], w[j], b[j]);
                            hat_r[8 * v + j] = fmaf(g[8 * v + j], a[8 * v + j], hat_r[8 * v + j]);
                        }
                    }
                    get(stage, IN_DR, v, row, D + 8 * v);
                    if (p.dn) {
                        get(stage, IN_DN, v, row, in8);
                        param8<VEC>(p.w_pre, 1.0f, v, t, threads, p.d, w);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int i = 8 * v + j;
                            hat_r[i] = (hat_r[i] - st.z) * st.w;
                            sum_pre_w[i] = fmaf(in8[j], hat_r[i], sum_pre_w[i]);
                            sum_pre_b[i] += in8[j];
                            q[i] = in8[j] * w[j];
                            s[0] += q[i];
                            s[1] = fmaf(q[i], hat_r[i], s[1]);
                        }
                    }
                }
                if (p.dn) {
                    row_sum<2>(s, slots, t, threads, id);
                    float* const swap = slots; slots = other; other = swap;
                    const float m0 = p.pre == BIGMAC_NORM_LAYER ? s[0] * p.inv_d : 0.0f, m1 = s[1] * p.inv_d;
#pragma unroll
                    for (int i = 0; i < 8 * NV; ++i) D[i] = fmaf(st.w, q[i] - m0 - hat_r[i] * m1, D[i]);
                }
            }
            if (p.dx) {
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float o[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[j] = p.rho * D[8 * v + j];
                    store8<T, VEC>((T*)p.dx + row * p.dx_ld, v, t, threads, p.d, o);
                }
            }
            if (!p.y) continue;
            if (p.dgate && p.gate_kind == BIGMAC_GATE_FULL) {
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float o[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[j] = D[8 * v + j] * a[8 * v + j];
                    store8<T, VEC>((T*)p.dgate + row * p.dgate_ld, v, t, threads, p.d, o);
                }
            }
            // sums of p and p hat, and of D a for a gate of the row; the channel gate's factor joins the column sums at the end
            float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float w[8];
                param8<VEC>(p.w_post, 1.0f, v, t, threads, p.d, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int i = 8 * v + j;
                    if (column<VEC>(v, j, t, threads) >= p.d) { D[i] = 0.0f; continue; }
                    const float Dg = D[i] * g[i], Ds = p.gate_kind == BIGMAC_GATE_CHANNEL ? D[i] : Dg;
                    sum_post_w[i] = fmaf(Ds, hat[i], sum_post_w[i]);
                    sum_post_b[i] += Ds;
                    s[2] = fmaf(D[i], a[i], s[2]);
                    D[i] = Dg * w[j];                                  // p
                    s[0] += D[i];
                    s[1] = fmaf(D[i], hat[i], s[1]);
                }
            }
            row_sum<3>(s, slots, t, threads, id);
            float* const swap = slots; slots = other; other = swap;
            if (p.dgate && p.gate_kind == BIGMAC_GATE_TOKEN && t == 0) ((float*)p.dgate)[row] = s[2];
            if (p.dy) {
                const float m0 = p.post == BIGMAC_NORM_LAYER ? s[0] * p.inv_d : 0.0f, m1 = s[1] * p.inv_d;
                const bool normed = p.post != BIGMAC_NORM_NONE;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float o[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int i = 8 * v + j;
                        o[j] = normed ? st.y * (D[i] - m0 - hat[i] * m1) : D[i];
                    }
                    store8<T, VEC>((T*)p.dy + row * p.dy_ld, v, t, threads, p.d, o);
                }
            }
        }
        if (VEC) asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
    if (!p.partial) return;
    // the block's sums: those of its rows of threads, in order (shared memory as [groups][d] floats, one quantity after the other)
    float* tile = (float*)ring;
#pragma unroll 1
    for (int which = 0; which < 4; ++which) {
        __syncthreads();
        if (working) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int c = column<VEC>(v, j, t, threads);
                    const float value = which == 0 ? sum_post_w[8 * v + j] : which == 1 ? sum_post_b[8 * v + j] : which == 2 ? sum_pre_w[8 * v + j] : sum_pre_b[8 * v + j];
                    if (c < p.d) tile[(size_t)group * p.d + c] = value;
                }
        }
        __syncthreads();
        float* out = p.partial + ((size_t)blockIdx.x * 4 + which) * p.d;
        for (int c = threadIdx.x; c < p.d; c += kBwdThreads) {
            float sum = 0.0f;
            for (int i = 0; i < groups; ++i) sum += tile[(size_t)i * p.d + c];
            out[c] = sum;
        }
    }
}

struct ParamGrads {
    float *dw_post, *db_post, *dw_pre, *db_pre, *dgate;               // dgate: of a channel gate
    const float *w_post, *b_post, *gate;                              // gate: a channel gate
    int accumulate;
};

// Column sums of the blocks' parts, 32 columns a block; the parts are added in a fixed order.
__global__ void __launch_bounds__(1024) residual_norm_sums_kernel(const float* __restrict__ partial, int parts, int d, const ParamGrads g) {
    __shared__ float tile[32][33];
    grid_dependency_launch();
    grid_dependency_wait();
    const int c = blockIdx.x * 32 + threadIdx.x, which = blockIdx.y;
    auto total = [&](int w) {
        float s = 0.0f;
        if (c < d) for (int i = threadIdx.y; i < parts; i += 32) s += partial[((size_t)i * 4 + w) * d + c];
        __syncthreads();
        tile[threadIdx.y][threadIdx.x] = s;
        __syncthreads();
        s = 0.0f;
        if (threadIdx.y == 0)
            for (int i = 0; i < 32; ++i) s += tile[i][threadIdx.x];
        return s;                                                      // in row 0 of the block
    };
    auto put = [&](float* to, float v) { if (to && threadIdx.y == 0 && c < d) to[c] = g.accumulate ? to[c] + v : v; };
    if (which == 1) {
        const float w = total(2), b = total(3);
        put(g.dw_pre, w);
        put(g.db_pre, b);
    } else {
        const float w = total(0), b = total(1);
        const float gate = g.gate && c < d ? g.gate[c] : 1.0f;
        put(g.dw_post, gate * w);
        put(g.db_post, gate * b);
        if (g.dgate && c < d) put(g.dgate, (g.w_post ? g.w_post[c] : 1.0f) * w + (g.b_post ? g.b_post[c] * b : 0.0f));
    }
}

Params params_of(const ResNorm& a) {
    const bigmac_residual_norm_t& q = *a.q;
    Params p{};
    p.x = q.x.p; p.y = q.y.p; p.gate = q.gate.p; p.dr = q.dr.p; p.dn = q.dn.p;
    p.r = q.r.p; p.n = q.n.p; p.dx = q.dx.p; p.dy = q.dy.p; p.dgate = q.dgate.p;
    p.x_ld = q.x.ld; p.y_ld = q.y.ld; p.gate_ld = q.gate.ld; p.dr_ld = q.dr.ld; p.dn_ld = q.dn.ld;
    p.r_ld = q.r.ld; p.n_ld = q.n.ld; p.dx_ld = q.dx.ld; p.dy_ld = q.dy.ld; p.dgate_ld = q.dgate.ld;
    p.w_post = q.w_post; p.b_post = q.b_post; p.w_pre = q.w_pre; p.b_pre = q.b_pre;
    p.stats = (float4*)q.stats;
    p.rho = q.residual_scale; p.post_eps = q.post_eps; p.pre_eps = q.pre_eps; p.inv_d = 1.0f / (float)q.d;
    p.T = a.T; p.d = q.d; p.post = q.post_kind; p.pre = q.pre_kind; p.gate_kind = q.gate_kind;
    return p;
}

// Threads of a row of d columns, 8 nv of them each: whole warps.
int threads_of(int d, int nv) { return (d + 8 * nv * 32 - 1) / (8 * nv * 32) * 32; }

template <typename T, int NV>
cudaError_t forward(const ResNorm& a, cudaStream_t stream) {
    const int threads = threads_of(a.q->d, NV), rows = threads == 32 ? 8 : 1;      // short rows: a warp each, eight a block
    const int64_t grid = ((int64_t)a.T + rows - 1) / rows;
    return a.vec ? launch_chained(residual_norm_kernel<T, NV, true>, (int)grid, rows * threads, 0, stream, params_of(a), threads)
                 : launch_chained(residual_norm_kernel<T, NV, false>, (int)grid, rows * threads, 0, stream, params_of(a), threads);
}

template <typename T, int NV, bool VEC, int STAGES>
cudaError_t backward(const ResNorm& a, float* partial, int grid, cudaStream_t stream) {
    auto kernel = residual_norm_bwd_kernel<T, NV, VEC, STAGES>;
    const int threads = threads_of(a.q->d, NV), groups = kBwdThreads / threads;
    size_t smem = VEC ? (size_t)STAGES * IN_COUNT * NV * sizeof(T) / 2 * kBwdThreads * 16 : 0;
    const size_t tile = (size_t)groups * a.q->d * sizeof(float);
    if (tile > smem) smem = tile;
    static PerDeviceOnce once;
    int dev;
    if (once.needed(&dev)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
        if (e != cudaSuccess) return e;
        once.mark(dev);
    }
    Params p = params_of(a);
    p.partial = partial;
    return launch_chained(kernel, grid, kBwdThreads, smem, stream, p, threads);
}

// Columns a thread of the backward kernel has, in pieces of 8.
int bwd_pieces(int d) { return d > 8 * kBwdThreads ? 2 : 1; }

}  // namespace

int residual_norm_parts(int T, int d) {
    const int groups = kBwdThreads / threads_of(d, bwd_pieces(d)), sms = gemm_tc_sm_count();
    const int64_t want = ((int64_t)T + groups - 1) / groups;
    return (int)(want < sms ? want : sms);
}

cudaError_t launch_residual_norm_forward(const ResNorm& a, cudaStream_t stream) {
    if (a.T == 0) return cudaSuccess;
    const bool few = a.T < 2 * gemm_tc_sm_count();
    const int d = a.q->d;
    if (a.q->dtype == BIGMAC_BF16) return few && d > 256 ? forward<__nv_bfloat16, 1>(a, stream) : d > 256 ? forward<__nv_bfloat16, 4>(a, stream) : forward<__nv_bfloat16, 1>(a, stream);
    return few || d <= 256 ? forward<float, 1>(a, stream) : forward<float, 2>(a, stream);
}

cudaError_t launch_residual_norm_backward(const ResNorm& a, float* partial, int accumulate, cudaStream_t stream) {
    const bigmac_residual_norm_t& q = *a.q;
    float* channel = q.gate_kind == BIGMAC_GATE_CHANNEL ? (float*)q.dgate.p : nullptr;
    const bool post = q.y.p && (q.dw_post || q.db_post || channel), pre = q.dn.p && (q.dw_pre || q.db_pre);
    const bool any = q.dw_post || q.db_post || q.dw_pre || q.db_pre || channel;
    int parts = 0;
    if (a.T > 0) {
        parts = residual_norm_parts(a.T, q.d);
        float* to = post || pre ? partial : nullptr;
        cudaError_t e;
        const bool wide = bwd_pieces(q.d) == 2;
        if (q.dtype == BIGMAC_BF16)
            e = a.vec ? (wide ? backward<__nv_bfloat16, 2, true, 2>(a, to, parts, stream) : backward<__nv_bfloat16, 1, true, 4>(a, to, parts, stream))
                      : (wide ? backward<__nv_bfloat16, 2, false, 1>(a, to, parts, stream) : backward<__nv_bfloat16, 1, false, 1>(a, to, parts, stream));
        else
            e = a.vec ? (wide ? backward<float, 2, true, 1>(a, to, parts, stream) : backward<float, 1, true, 2>(a, to, parts, stream))
                      : (wide ? backward<float, 2, false, 1>(a, to, parts, stream) : backward<float, 1, false, 1>(a, to, parts, stream));
        if (e != cudaSuccess) return e;
    }
    if (!any) return cudaSuccess;
    // without rows, or without their source, the sums are zero: no parts
    ParamGrads g{q.dw_post, q.db_post, q.dw_pre, q.db_pre, channel, q.w_post, q.b_post, channel ? (const float*)q.gate.p : nullptr, accumulate};
    if (q.gate_kind == BIGMAC_GATE_CHANNEL) g.gate = (const float*)q.gate.p;
    return launch_chained(residual_norm_sums_kernel, dim3((q.d + 31) / 32, 2), dim3(32, 32), 0, stream, partial, post || pre ? parts : 0, q.d, g);
}

}  // namespace bigmac
