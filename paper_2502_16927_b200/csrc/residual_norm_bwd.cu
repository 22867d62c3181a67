// Backward of the joint of two blocks (formulas: residual_norm.cu).
//
// Bound by memory: x, y, dr, dn (and a full gate) in, dx, dy (and its gradient) out, every element once; r and both normalised rows are
// computed again from x, y and the four statistics of a row.
#include "residual_norm.cuh"

namespace bigmac {

using namespace resnorm;

namespace {

enum { IN_X = 0, IN_Y, IN_DR, IN_DN, IN_GATE, IN_COUNT };

// Persistent blocks of 512 threads, `threads` of them to a row, 8 NV columns a thread; a thread keeps the column sums of its
// columns over its rows.  RING: the inputs of the next rows are on their way to shared memory while a row is worked on, parameters stay there, a
// channel gate is part of them.  Without (rows of more than 4096 columns in fp32, with biases or off 16-byte boundaries): everything loaded when it is
// needed (4000 rows of 8192 265 us, with 90).
// GATE (of bigmac_gate_t, kNoBlock, kAnyGate) and DN are fixed at compile time for RING: with the choice at run time a row took twice the
// instructions.  BIAS: the sums that only biases need are kept, too; without them there is room for 16 columns a thread, and half the threads of a
// row are a third fewer instructions for it (16384 rows of 4096, RMS norms, a full gate: 219 us with 8 columns, 183 with 16).  There, what is needed again
// behind a sum is read again from shared memory; with 8 columns it is held in registers (16384 rows of 2048, LayerNorms: 101 us, read again 118).
template <typename T, int NV, int VEC, bool RING, int GATE, bool DN, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1) residual_norm_bwd_kernel(const Params p, int threads, int stages) {
    extern __shared__ __align__(16) uint8_t smem[];
    constexpr int SB = BIAS ? 4 * NV : 1;
    constexpr bool HOLD = NV == 1;
    constexpr int H = HOLD ? 4 : 1;
    __shared__ __align__(16) float sums[2][kThreads / 32][32];
    grid_dependency_launch();
    grid_dependency_wait();
    const int t = threadIdx.x % threads, group = threadIdx.x / threads, groups = kThreads / threads;
    const int first = (int)blockIdx.x * groups + group, step = (int)gridDim.x * groups;
    const bool working = group < groups;                               // threads that are no whole row rest
    Row at(sums[0][working ? group : 0], sums[1][working ? group : 0], t, threads, 1 + group);
    const int gate_kind = GATE == kAnyGate ? p.gate_kind : GATE;       // RING: a channel gate counts as none
    const bool has_y = GATE == kAnyGate ? p.y != nullptr : GATE != kNoBlock;
    const bool has_dn = GATE == kAnyGate ? p.dn != nullptr : DN;
    constexpr int COUNT = GATE == BIGMAC_GATE_FULL || GATE == kAnyGate ? IN_COUNT : IN_COUNT - 1;
    Ring<T, VEC, COUNT, NV> ring;
    ring.in[IN_X] = (const T*)p.x; ring.in[IN_Y] = (const T*)p.y; ring.in[IN_DR] = (const T*)p.dr; ring.in[IN_DN] = (const T*)p.dn;
    ring.ld[IN_X] = p.x_ld; ring.ld[IN_Y] = p.y_ld; ring.ld[IN_DR] = p.dr_ld; ring.ld[IN_DN] = p.dn_ld;
    ring.has[IN_X] = true; ring.has[IN_Y] = has_y; ring.has[IN_DR] = p.dr != nullptr; ring.has[IN_DN] = has_dn;
    if constexpr (COUNT == IN_COUNT) { ring.in[IN_GATE] = (const T*)p.gate; ring.ld[IN_GATE] = p.gate_ld; ring.has[IN_GATE] = gate_kind == BIGMAC_GATE_FULL; }
    auto get = [&](int stage, int which, int v, int row, f2* f) {
        if constexpr (RING) ring.get(stage, which, v, row, t, threads, f);
        else if (ring.has[which]) load8<T, VEC>(row_at(ring.in[which], row, ring.ld[which]), v, t, threads, p.d, f);
        else fill8(0.0f, f);
    };
    constexpr bool kShared = NV == 2;
    ParamStore<NV, kShared> par(smem, t, threads);                              // RING: w_post, w_pre, and with BIAS b_post
    enum { W_POST = 0, W_PRE = 1, B_POST = 2 };
    auto param = [&](int which, int v, f2* f) {
        if constexpr (RING) par.get(which, v, f);
        else param8<VEC>(which == W_POST ? p.w_post : which == W_PRE ? p.w_pre : p.b_post, which == B_POST ? 0.0f : 1.0f, v, t, threads, p.d, f);
    };
    auto gate8 = [&](int stage, int v, int row, float token, f2* f) {
        if (COUNT == IN_COUNT && gate_kind == BIGMAC_GATE_FULL) get(stage, COUNT - 1, v, row, f);
        else if (gate_kind == BIGMAC_GATE_CHANNEL) load8<float, VEC>((const float*)p.gate, v, t, threads, p.d, f);
        else fill8(token, f);
    };

    f2 sum_post_w[4 * NV], sum_pre_w[4 * NV], sum_post_b[SB], sum_pre_b[SB];
#pragma unroll
    for (int i = 0; i < 4 * NV; ++i) sum_post_w[i] = sum_pre_w[i] = pk(0.0f);
#pragma unroll
    for (int i = 0; i < SB; ++i) sum_post_b[i] = sum_pre_b[i] = pk(0.0f);

    if (working) {
        if constexpr (RING) {
            ring.init(smem + (BIAS ? 3 : 2) * param_bytes(kShared, threads, NV), group, stages, p);
            ring.start(first, step, t, threads);
#pragma unroll
            for (int v = 0; v < NV; ++v) {                             // every group of threads writes the same numbers
                f2 w[4], b[4];
                if (has_y) {
                    post_params<VEC>(p, v, t, threads, w, b);
                    par.put(W_POST, v, w);
                    if (BIAS) par.put(B_POST, v, b);
                }
                param8<VEC>(p.w_pre, 1.0f, v, t, threads, p.d, w);
                par.put(W_PRE, v, w);
            }
        }
        int stage = 0;
        const f2 rho = pk(p.rho);
        float4 next_stats = first < p.T ? p.stats[first] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int row = first; row < p.T; row += step) {
            const float4 st = next_stats;
            if (row + step < p.T) next_stats = p.stats[row + step];
            const float token = gate_kind == BIGMAC_GATE_TOKEN ? ((const float*)p.gate)[row] : 1.0f;
            if constexpr (RING) ring.next(stage, row, step, at);
            f2 hat[4 * NV], hat_r[4 * NV], D[4 * NV], s0 = pk(0.0f), s1 = pk(0.0f);
            f2 held_a[H], held_g[H], held_q[H], held_w[H];             // HOLD
            // r and, behind its norm, the sums of q = dn w_pre and q hat_r
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                f2 w[4], b[4], e[4], g[4];
                get(stage, IN_X, v, row, hat_r + 4 * v);
#pragma unroll
                for (int j = 0; j < 4; ++j) hat_r[4 * v + j] = mul2(rho, hat_r[4 * v + j]);
                if (has_y) {
                    get(stage, IN_Y, v, row, e);
                    param(W_POST, v, w);
                    if (BIAS) param(B_POST, v, b); else fill8(0.0f, b);
                    if (gate_kind != BIGMAC_GATE_NONE) gate8(stage, v, row, token, g);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int i = 4 * v + j;
                        hat[i] = mul2(add2(e[j], pk(-st.x)), pk(st.y));
                        const f2 a = BIAS ? fma2(hat[i], w[j], b[j]) : mul2(hat[i], w[j]);
                        hat_r[i] = gate_kind == BIGMAC_GATE_NONE ? add2(a, hat_r[i]) : fma2(g[j], a, hat_r[i]);
                        if (HOLD) { held_a[j % H] = a; held_g[j % H] = g[j]; held_w[j % H] = w[j]; }
                    }
                }
                if (HOLD) get(stage, IN_DR, v, row, D + 4 * v);
                if (has_dn) {
                    get(stage, IN_DN, v, row, e);
                    param(W_PRE, v, w);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int i = 4 * v + j;
                        hat_r[i] = mul2(add2(hat_r[i], pk(-st.z)), pk(st.w));
                        sum_pre_w[i] = fma2(e[j], hat_r[i], sum_pre_w[i]);
                        if (BIAS) sum_pre_b[BIAS ? i : 0] = add2(e[j], sum_pre_b[BIAS ? i : 0]);
                        const f2 q = mul2(e[j], w[j]);
                        if (HOLD) held_q[j % H] = q;
                        s0 = add2(s0, q);
                        s1 = fma2(q, hat_r[i], s1);
                    }
                }
            }
            float m0 = 0.0f, m1 = 0.0f;
            if (has_dn) {
                m0 = both(s0); m1 = both(s1);
                row_sum2(m0, m1, at);
                m0 = p.pre == BIGMAC_NORM_LAYER ? -m0 * p.inv_d : 0.0f;
                m1 *= -p.inv_d;
            }
            // D = dr + the norm's part; the sums of p = gate D w_post and p hat, and of D a for a gate of the row; a channel gate's factor joins the
            // column sums at the end
            s0 = s1 = pk(0.0f);
            f2 s2 = pk(0.0f);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                f2 w[4], b[4], e[4], g[4], o[4];
                if (!HOLD) get(stage, IN_DR, v, row, D + 4 * v);
                if (has_dn) {
                    if (!HOLD) {
                        get(stage, IN_DN, v, row, e);
                        param(W_PRE, v, w);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int i = 4 * v + j;
                        D[i] = fma2(pk(st.w), fma2(hat_r[i], pk(m1), HOLD ? add2(held_q[j % H], pk(m0)) : fma2(e[j], w[j], pk(m0))), D[i]);
                    }
                }
                if (p.dx) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[j] = mul2(rho, D[4 * v + j]);
                    store8<T, VEC>(row_at((T*)p.dx, row, p.dx_ld), v, t, threads, p.d, o);
                }
                if (!has_y) continue;
                if (HOLD) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) { w[j] = held_w[j % H]; g[j] = held_g[j % H]; }
                } else {
                    param(W_POST, v, w);
                    if (gate_kind != BIGMAC_GATE_NONE) gate8(stage, v, row, token, g);
                }
                if (!RING) cut8<VEC>(v, t, threads, p.d, D + 4 * v);       // RING: w_post and b_post are zeros there
                if ((gate_kind == BIGMAC_GATE_FULL && p.dgate) || gate_kind == BIGMAC_GATE_TOKEN) {
                    if (BIAS && !HOLD) param(B_POST, v, b); else fill8(0.0f, b);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int i = 4 * v + j;
                        o[j] = mul2(D[i], HOLD ? held_a[j % H] : BIAS ? fma2(hat[i], w[j], b[j]) : mul2(hat[i], w[j]));
                        if (gate_kind == BIGMAC_GATE_TOKEN) s2 = add2(s2, o[j]);
                    }
                    if (gate_kind == BIGMAC_GATE_FULL) store8<T, VEC>(row_at((T*)p.dgate, row, p.dgate_ld), v, t, threads, p.d, o);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = 4 * v + j;
                    const f2 Dg = gate_kind == BIGMAC_GATE_NONE ? D[i] : mul2(D[i], g[j]), Ds = gate_kind == BIGMAC_GATE_CHANNEL ? D[i] : Dg;
                    sum_post_w[i] = fma2(Ds, hat[i], sum_post_w[i]);
                    if (BIAS) sum_post_b[BIAS ? i : 0] = add2(Ds, sum_post_b[BIAS ? i : 0]);
                    D[i] = mul2(Dg, w[j]);                             // p
                    s0 = add2(s0, D[i]);
                    s1 = fma2(D[i], hat[i], s1);
                }
            }
            if (has_y) {
                if (gate_kind == BIGMAC_GATE_TOKEN && p.dgate) {
                    const float sum = row_sum(both(s2), at);
                    if (t == 0) ((float*)p.dgate)[row] = sum;
                }
                if (p.dy) {
                    if (p.post != BIGMAC_NORM_NONE) {
                        m0 = both(s0); m1 = both(s1);
                        row_sum2(m0, m1, at);
                        m0 = p.post == BIGMAC_NORM_LAYER ? -m0 * p.inv_d : 0.0f;
                        m1 *= -p.inv_d;
#pragma unroll
                        for (int i = 0; i < 4 * NV; ++i) D[i] = mul2(pk(st.y), fma2(hat[i], pk(m1), add2(D[i], pk(m0))));
                    }
#pragma unroll
                    for (int v = 0; v < NV; ++v) store8<T, VEC>(row_at((T*)p.dy, row, p.dy_ld), v, t, threads, p.d, D + 4 * v);
                }
            }
            if constexpr (RING) stage = stage + 1 == stages ? 0 : stage + 1;
        }
        if constexpr (RING) wait_groups(0);
    }
    if (!p.partial) return;
    // the block's sums: those of its rows of threads, in order (shared memory as [groups][d] floats, one quantity after the other).  Places worked
    // out again: the loop above has no register for them
    int tid;
    asm volatile("mov.u32 %0, %%tid.x;" : "=r"(tid));
    const int own = tid % threads, own_group = tid / threads, all = kThreads / threads;
    float* tile = (float*)smem;
#pragma unroll
    for (int which = 0; which < 4; which += BIAS ? 1 : 2) {
        float* out = p.partial + ((size_t)blockIdx.x * 4 + which) * p.d;
        const f2* mine = which == 0 ? sum_post_w : which == 1 ? sum_post_b : which == 2 ? sum_pre_w : sum_pre_b;
        __syncthreads();
        if (own_group < all) {
#pragma unroll
            for (int v = 0; v < NV; ++v) store8<float, VEC>(tile + (size_t)own_group * p.d, v, own, threads, p.d, mine + 4 * v);
        }
        __syncthreads();
        for (int c = tid; c < p.d; c += kThreads) {
            float sum = 0.0f;
            for (int i = 0; i < all; ++i) sum += tile[(size_t)i * p.d + c];
            out[c] = sum;
        }
    }
}

struct ParamGrads {
    float *dw_post, *db_post, *dw_pre, *db_pre, *dgate;               // dgate: of a channel gate
    const float *w_post, *b_post, *gate;                              // gate: a channel gate
    int accumulate, bias;                                             // bias: the parts hold the sums that only biases need
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
        const float w = total(2), b = g.bias ? total(3) : 0.0f;
        put(g.dw_pre, w);
        put(g.db_pre, b);
    } else {
        const float w = total(0), b = g.bias ? total(1) : 0.0f;
        const float gate = g.gate && c < d ? g.gate[c] : 1.0f;
        put(g.dw_post, gate * w);
        put(g.db_post, gate * b);
        if (g.dgate && c < d) put(g.dgate, (g.w_post ? g.w_post[c] : 1.0f) * w + (g.b_post ? g.b_post[c] * b : 0.0f));
    }
}

constexpr size_t kBwdSmem = 214 * 1024;                                // and 4 KB for sums

template <typename T, int NV, int VEC, bool RING, int GATE, bool DN, bool BIAS>
cudaError_t backward(const ResNorm& a, float* partial, int grid, cudaStream_t stream) {
    auto kernel = residual_norm_bwd_kernel<T, NV, VEC, RING, GATE, DN, BIAS>;
    const int threads = threads_of(a.q->d, NV), groups = kThreads / threads;
    size_t smem = (size_t)groups * a.q->d * sizeof(float);             // the block's sums at the end
    int stages = 0;
    if (RING) {
        const size_t stage = stage_bytes(VEC, a.q->d, (int)sizeof(T), groups, GATE == BIGMAC_GATE_FULL ? IN_COUNT : IN_COUNT - 1, NV), par = (BIAS ? 3 : 2) * param_bytes(NV == 2, threads, NV);
        stages = (int)((kBwdSmem - par) / stage > 4 ? 4 : (kBwdSmem - par) / stage);
        if (stages < 1) return cudaErrorInvalidValue;
        if (par + stages * stage > smem) smem = par + stages * stage;
    }
    static PerDeviceOnce once;
    int dev;
    if (once.needed(&dev)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kBwdSmem);
        if (e != cudaSuccess) return e;
        once.mark(dev);
    }
    Params p = params_of(a);
    p.partial = partial;
    return launch_chained(kernel, grid, kThreads, smem, stream, p, threads, stages);
}
// Do the sums that only biases need matter?  (A channel gate's gradient has b_post in it.)
bool wants_bias(const bigmac_residual_norm_t& q) { return q.b_post || q.db_post || q.db_pre; }
// Columns a thread has, in pieces of 8.  (Rows off 16-byte boundaries with 16 columns a thread spill registers: 8000 rows of 2999 158 us, 198.)
int bwd_pieces(const ResNorm& a) {
    if (a.q->d > 8 * kThreads) return 2;
    return a.vec && !wants_bias(*a.q) && a.q->dtype == BIGMAC_BF16 && a.q->d > 256 ? 2 : 1;
}
int blocks_of(int T, int d, int nv) {
    const int groups = kThreads / threads_of(d, nv), sms = gemm_tc_sm_count();
    const int64_t want = ((int64_t)T + groups - 1) / groups;
    return (int)(want < sms ? want : sms);
}
template <typename T, int NV, int VEC, bool DN, bool BIAS>
cudaError_t backward_by_gate(const ResNorm& a, float* partial, int grid, cudaStream_t stream) {
    if (!a.q->y.p) return backward<T, NV, VEC, true, kNoBlock, DN, BIAS>(a, partial, grid, stream);
    switch (a.q->gate_kind) {
        case BIGMAC_GATE_TOKEN: return backward<T, NV, VEC, true, BIGMAC_GATE_TOKEN, DN, BIAS>(a, partial, grid, stream);
        case BIGMAC_GATE_FULL: return backward<T, NV, VEC, true, BIGMAC_GATE_FULL, DN, BIAS>(a, partial, grid, stream);
        default: return backward<T, NV, VEC, true, BIGMAC_GATE_NONE, DN, BIAS>(a, partial, grid, stream);
    }
}
template <typename T>
cudaError_t backward_any(const ResNorm& a, float* partial, int grid, cudaStream_t stream) {
    const bool dn = a.q->dn.p != nullptr;
    if (a.q->d > 8 * kThreads && (!a.vec || sizeof(T) == 4 || wants_bias(*a.q)))
        return a.vec ? backward<T, 2, kVecOf<T>, false, kAnyGate, true, true>(a, partial, grid, stream) : backward<T, 2, kAlternate, false, kAnyGate, true, true>(a, partial, grid, stream);
    if constexpr (sizeof(T) == 2)
        if (bwd_pieces(a) == 2)
            return dn ? backward_by_gate<T, 2, kVecOf<T>, true, false>(a, partial, grid, stream) : backward_by_gate<T, 2, kVecOf<T>, false, false>(a, partial, grid, stream);
    if (a.vec) return dn ? backward_by_gate<T, 1, kVecOf<T>, true, true>(a, partial, grid, stream) : backward_by_gate<T, 1, kVecOf<T>, false, true>(a, partial, grid, stream);
    return dn ? backward_by_gate<T, 1, kAlternate, true, true>(a, partial, grid, stream) : backward_by_gate<T, 1, kAlternate, false, true>(a, partial, grid, stream);
}

}  // namespace

int residual_norm_parts(int T, int d) { return blocks_of(T, d, d > 8 * kThreads ? 2 : 1); }

cudaError_t launch_residual_norm_backward(const ResNorm& a, float* partial, int accumulate, cudaStream_t stream) {
    const bigmac_residual_norm_t& q = *a.q;
    float* channel = q.gate_kind == BIGMAC_GATE_CHANNEL ? (float*)q.dgate.p : nullptr;
    const bool post = q.y.p && (q.dw_post || q.db_post || channel), pre = q.dn.p && (q.dw_pre || q.db_pre);
    const bool any = q.dw_post || q.db_post || q.dw_pre || q.db_pre || channel;
    int parts = 0;
    if (a.T > 0) {
        parts = blocks_of(a.T, q.d, bwd_pieces(a));
        float* to = post || pre ? partial : nullptr;
        cudaError_t e;
        if (q.dtype == BIGMAC_BF16) e = backward_any<__nv_bfloat16>(a, to, parts, stream);
        else e = backward_any<float>(a, to, parts, stream);
        if (e != cudaSuccess) return e;
    }
    if (!any) return cudaSuccess;
    // without rows, or without their source, the sums are zero: no parts
    const float* gate = q.gate_kind == BIGMAC_GATE_CHANNEL ? (const float*)q.gate.p : nullptr;
    const ParamGrads g{q.dw_post, q.db_post, q.dw_pre, q.db_pre, channel, q.w_post, q.b_post, gate, accumulate, wants_bias(q)};
    return launch_chained(residual_norm_sums_kernel, dim3((q.d + 31) / 32, 2), dim3(32, 32), 0, stream, partial, post || pre ? parts : 0, q.d, g);
}

}  // namespace bigmac
