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
// dx, dy out.  Both read every tensor once: a row lies in the registers of one to 16 warps, which share its sums.
#include "residual_norm.cuh"

namespace bigmac {

using namespace resnorm;

namespace {

// Few rows, fp32 ones on 16-byte boundaries however many, and rows of more than 4096 columns off them: one row to `threads` threads, 8 NV columns
// each.  Rows of a warp may share a block, longer ones have one for themselves.
template <typename T, int NV, int VEC>
__global__ void __launch_bounds__(kThreads, NV == 1 ? 2 : 1) residual_norm_kernel(const Params p, int threads) {
    __shared__ __align__(16) float sums[2][32];
    grid_dependency_launch();
    grid_dependency_wait();
    const int in_block = threads == 32 ? threadIdx.x >> 5 : 0;
    Row at(sums[0], sums[1], threads == 32 ? (int)threadIdx.x & 31 : (int)threadIdx.x, threads, 1);
    const int t = at.t;
    const int row = (int)blockIdx.x * (threads == 32 ? (int)blockDim.x >> 5 : 1) + in_block;
    if (row >= p.T) return;
    f2 r[4 * NV], y[4 * NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) load8<T, VEC>(row_at((const T*)p.x, row, p.x_ld), v, t, threads, p.d, r + 4 * v);
    float4 st = make_float4(0.0f, 1.0f, 0.0f, 1.0f);
    const f2 rho = pk(p.rho);
    if (p.y) {
#pragma unroll
        for (int v = 0; v < NV; ++v) load8<T, VEC>(row_at((const T*)p.y, row, p.y_ld), v, t, threads, p.d, y + 4 * v);
        f2 g[4 * NV];
        if (p.gate_kind == BIGMAC_GATE_FULL) {
#pragma unroll
            for (int v = 0; v < NV; ++v) load8<T, VEC>(row_at((const T*)p.gate, row, p.gate_ld), v, t, threads, p.d, g + 4 * v);
        } else if (p.gate_kind == BIGMAC_GATE_CHANNEL) {
#pragma unroll
            for (int v = 0; v < NV; ++v) load8<float, VEC>((const float*)p.gate, v, t, threads, p.d, g + 4 * v);
        } else {
            const float token = p.gate_kind == BIGMAC_GATE_TOKEN ? ((const float*)p.gate)[row] : 1.0f;
#pragma unroll
            for (int v = 0; v < NV; ++v) fill8(token, g + 4 * v);
        }
        row_stats<NV, VEC>(p.post, y, p.post_eps, p, at, st.x, st.y);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            f2 w[4], b[4];
            param8<VEC>(p.w_post, 1.0f, v, t, threads, p.d, w);
            param8<VEC>(p.b_post, 0.0f, v, t, threads, p.d, b);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = 4 * v + j;
                const f2 a = fma2(mul2(add2(y[i], pk(-st.x)), pk(st.y)), w[j], b[j]);
                r[i] = fma2(rho, r[i], mul2(g[i], a));
            }
            cut8<VEC>(v, t, threads, p.d, r + 4 * v);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) r[i] = mul2(r[i], rho);
    }
    if (p.r) {
#pragma unroll
        for (int v = 0; v < NV; ++v) store8<T, VEC>(row_at((T*)p.r, row, p.r_ld), v, t, threads, p.d, r + 4 * v);
    }
    if (p.n) {
        row_stats<NV, VEC>(p.pre, r, p.pre_eps, p, at, st.z, st.w);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            f2 w[4], b[4];
            param8<VEC>(p.w_pre, 1.0f, v, t, threads, p.d, w);
            param8<VEC>(p.b_pre, 0.0f, v, t, threads, p.d, b);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = fma2(mul2(add2(r[4 * v + j], pk(-st.z)), pk(st.w)), w[j], b[j]);
            store8<T, VEC>(row_at((T*)p.n, row, p.n_ld), v, t, threads, p.d, w);
        }
    }
    if (p.stats && t == 0) p.stats[row] = st;
}

// Many rows: persistent blocks of 512 threads, `threads` of them to a row, 8 NV columns a thread: two blocks on an SM with eight columns, one with 16.  A
// block a row spent 2 us of an SM on a row of 4096 columns whatever its type, all of it latencies one after the other (loads, sums, parameters,
// sums); here the next rows are on their way meanwhile and the parameters stay in shared memory (4000 rows of 8192: 100 us a block a row, 53 here).
template <int NV>
constexpr bool kSharedParams = NV == 2;                                // 16 columns a thread: a block's rows read one copy, which leaves room for more rows
template <typename T, int NV, int VEC, int GATE>
__global__ void __launch_bounds__(kThreads, NV == 1 ? 2 : 1) residual_norm_rows_kernel(const Params p, int threads, int stages, int vectors) {
    extern __shared__ __align__(16) uint8_t smem[];
    constexpr int COUNT = GATE == kNoBlock ? 1 : GATE == BIGMAC_GATE_FULL ? 3 : 2;
    __shared__ __align__(16) float sums[2][kThreads / 32][32];
    grid_dependency_launch();
    grid_dependency_wait();
    const int t = threadIdx.x % threads, group = threadIdx.x / threads, groups = kThreads / threads;
    if (group >= groups) return;                                       // threads that are no whole row
    const int first = (int)blockIdx.x * groups + group, step = (int)gridDim.x * groups;
    Row at(sums[0][group], sums[1][group], t, threads, 1 + group);
    Ring<T, VEC, COUNT, NV> ring;
    const void* const in[3] = {p.x, p.y, p.gate};
    const int ld[3] = {p.x_ld, p.y_ld, p.gate_ld};
#pragma unroll
    for (int i = 0; i < COUNT; ++i) { ring.in[i] = (const T*)in[i]; ring.ld[i] = ld[i]; ring.has[i] = true; }
    ring.init(smem + vectors * param_bytes(kSharedParams<NV>, threads, NV), group, stages, p);
    ring.template start<VEC>(first, step, t, threads);
    // vectors 0, 1: w and b of the norm before, 2, 3: of the one behind; b only with `vectors` = 4.
    ParamStore<NV, kSharedParams<NV>> par(smem, t, threads);
    const int pre = vectors / 2;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        f2 w[4], b[4];
        if (GATE != kNoBlock) {
            post_params<VEC>(p, v, t, threads, w, b);
            par.put(0, v, w);
            if (vectors == 4) par.put(1, v, b);
        }
        param8<VEC>(p.w_pre, 1.0f, v, t, threads, p.d, w);
        par.put(pre, v, w);
        if (vectors == 4) {
            param8<VEC>(p.b_pre, 0.0f, v, t, threads, p.d, b);
            par.put(3, v, b);
        }
    }
    int stage = 0;
    const f2 rho = pk(p.rho);
    for (int row = first; row < p.T; row += step) {
        const float token = GATE == BIGMAC_GATE_TOKEN ? ((const float*)p.gate)[row] : 1.0f;
        if constexpr (VEC) ring.arrived();
        else ring.next(stage, row, step, at);
        f2 r[4 * NV];
        float4 st = make_float4(0.0f, 1.0f, 0.0f, 1.0f);
#pragma unroll
        for (int v = 0; v < NV; ++v) ring.get(stage, 0, v, row, t, threads, r + 4 * v);
#pragma unroll
        for (int j = 0; j < 4 * NV; ++j) r[j] = mul2(rho, r[j]);
        if constexpr (GATE != kNoBlock) {
            f2 y[4 * NV];
#pragma unroll
            for (int v = 0; v < NV; ++v) ring.get(stage, 1, v, row, t, threads, y + 4 * v);
            row_stats<NV, VEC>(p.post, y, p.post_eps, p, at, st.x, st.y);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                f2 w[4], b[4], g[4];
                if constexpr (GATE == BIGMAC_GATE_FULL) ring.get(stage, 2, v, row, t, threads, g);
                par.get(0, v, w);
                if (vectors == 4) par.get(1, v, b); else fill8(0.0f, b);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = 4 * v + j;
                    const f2 a = fma2(mul2(add2(y[i], pk(-st.x)), pk(st.y)), w[j], b[j]);
                    r[i] = GATE == BIGMAC_GATE_FULL ? fma2(g[j], a, r[i]) : GATE == BIGMAC_GATE_TOKEN ? fma2(pk(token), a, r[i]) : add2(a, r[i]);
                }
            }
        }
        if constexpr (VEC) ring.again(stage, row, step, at);
        if (p.r) {
#pragma unroll
            for (int v = 0; v < NV; ++v) store8<T, VEC>(row_at((T*)p.r, row, p.r_ld), v, t, threads, p.d, r + 4 * v);
        }
        if (p.n) {
            row_stats<NV, VEC>(p.pre, r, p.pre_eps, p, at, st.z, st.w);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                f2 w[4], b[4];
                par.get(pre, v, w);
                if (vectors == 4) par.get(3, v, b); else fill8(0.0f, b);
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = fma2(mul2(add2(r[4 * v + j], pk(-st.z)), pk(st.w)), w[j], b[j]);
                store8<T, VEC>(row_at((T*)p.n, row, p.n_ld), v, t, threads, p.d, w);
            }
        }
        if (p.stats && t == 0) p.stats[row] = st;
        stage = stage + 1 == stages ? 0 : stage + 1;
    }
    wait_groups(0);
}

template <typename T, int NV, int VEC>
cudaError_t one_row_a_block(const ResNorm& a, cudaStream_t stream) {
    const int threads = threads_of(a.q->d, NV), rows = threads == 32 ? (a.T < 8 * gemm_tc_sm_count() ? 1 : 8) : 1;
    if (threads > kThreads) return cudaErrorInvalidValue;             // the room for a row's sums is 16 warps'
    const int64_t grid = ((int64_t)a.T + rows - 1) / rows;
    return launch_chained(residual_norm_kernel<T, NV, VEC>, (int)grid, rows * threads, 0, stream, params_of(a), threads);
}

constexpr size_t kRowsSmem = 108 * 1024;                               // of a block, two to an SM (and 4 KB for sums)

template <typename T, int NV, int VEC, int GATE>
cudaError_t persistent(const ResNorm& a, cudaStream_t stream) {
    auto kernel = residual_norm_rows_kernel<T, NV, VEC, GATE>;
    const int threads = threads_of(a.q->d, NV), groups = kThreads / threads, count = GATE == kNoBlock ? 1 : GATE == BIGMAC_GATE_FULL ? 3 : 2;
    const int vectors = a.q->b_post || a.q->b_pre ? 4 : 2;
    const size_t stage = stage_bytes(VEC, a.q->d, (int)sizeof(T), groups, count, NV), par = vectors * param_bytes(kSharedParams<NV>, threads, NV), left = (NV == 1 ? 1 : 2) * kRowsSmem - par;
    const int stages = (int)(left / stage < 1 ? 1 : left / stage > 4 ? 4 : left / stage);
    static PerDeviceOnce once;
    int dev;
    if (once.needed(&dev)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * (int)kRowsSmem);
        if (e != cudaSuccess) return e;
        once.mark(dev);
    }
    const int64_t want = ((int64_t)a.T + groups - 1) / groups, most = (NV == 1 ? 2 : 1) * (int64_t)gemm_tc_sm_count();
    return launch_chained(kernel, (int)(want < most ? want : most), kThreads, par + stages * stage, stream, params_of(a), threads, stages, vectors);
}
template <typename T, int NV, int VEC>
cudaError_t persistent_by_gate(const ResNorm& a, cudaStream_t stream) {
    if (!a.q->y.p) return persistent<T, NV, VEC, kNoBlock>(a, stream);
    switch (a.q->gate_kind) {
        case BIGMAC_GATE_TOKEN: return persistent<T, NV, VEC, BIGMAC_GATE_TOKEN>(a, stream);
        case BIGMAC_GATE_FULL: return persistent<T, NV, VEC, BIGMAC_GATE_FULL>(a, stream);
        default: return persistent<T, NV, VEC, BIGMAC_GATE_NONE>(a, stream);
    }
}
// Columns a thread of the persistent blocks has, in pieces of eight: 16 are half the threads, and so half the instructions for the sums, of a row (us with
// eight / 16: 16384 x 4096 RMS, a full gate 114 / 107, 16384 x 2048 LayerNorms 69 / 63, 8000 x 1357 then 51 / 45, but 8000 x 1104 25.5 / 26.3).
template <typename T>
cudaError_t forward(const ResNorm& a, cudaStream_t stream) {
    const int d = a.q->d;
    const bool wide = d > 8 * kThreads, many = a.T > (int64_t)2 * gemm_tc_sm_count() * (wide ? 1 : kThreads / threads_of(d, 1)), pairs = d > 1280;
    if constexpr (sizeof(T) == 2)
        if (many && a.vec) return pairs ? persistent_by_gate<T, 2, kNeighbours>(a, stream) : persistent_by_gate<T, 1, kNeighbours>(a, stream);
    if (!a.vec) {
        if (!many || wide) return one_row_a_block<T, 2, kAlternate>(a, stream);
        return pairs ? persistent_by_gate<T, 2, kAlternate>(a, stream) : persistent_by_gate<T, 1, kAlternate>(a, stream);
    }
    return wide || (sizeof(T) == 4 && many) ? one_row_a_block<T, 2, kVecOf<T>>(a, stream) : one_row_a_block<T, 1, kVecOf<T>>(a, stream);
}

}  // namespace

Params resnorm::params_of(const ResNorm& a) {
    const bigmac_residual_norm_t& q = *a.q;
    Params p{};
    p.x = q.x.p; p.y = q.y.p; p.gate = q.gate.p; p.dr = q.dr.p; p.dn = q.dn.p;
    p.r = q.r.p; p.n = q.n.p; p.dx = q.dx.p; p.dy = q.dy.p; p.dgate = q.dgate.p;
    p.x_ld = (int)q.x.ld; p.y_ld = (int)q.y.ld; p.gate_ld = (int)q.gate.ld; p.dr_ld = (int)q.dr.ld; p.dn_ld = (int)q.dn.ld;
    p.r_ld = (int)q.r.ld; p.n_ld = (int)q.n.ld; p.dx_ld = (int)q.dx.ld; p.dy_ld = (int)q.dy.ld; p.dgate_ld = (int)q.dgate.ld;
    p.w_post = q.w_post; p.b_post = q.b_post; p.w_pre = q.w_pre; p.b_pre = q.b_pre;
    p.stats = (float4*)q.stats;
    p.rho = q.residual_scale; p.post_eps = q.post_eps; p.pre_eps = q.pre_eps; p.inv_d = 1.0f / (float)q.d;
    p.T = a.T; p.d = q.d; p.post = q.post_kind; p.pre = q.pre_kind; p.gate_kind = q.gate_kind;
    return p;
}

cudaError_t launch_residual_norm_forward(const ResNorm& a, cudaStream_t stream) {
    if (a.T == 0) return cudaSuccess;
    return a.q->dtype == BIGMAC_BF16 ? forward<__nv_bfloat16>(a, stream) : forward<float>(a, stream);
}

}  // namespace bigmac
