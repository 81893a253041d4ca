// Linear attention with a decay for each head (deer_linattn, deer_linattn_adjoint,
// deer_linattn_step).
//
// The recurrence S_t = a_t S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t and its three large gradients
// are the same walk with the operands in other places:
//   o  : q, k, v  forwards                 dq : g, v, k  forwards (the state is S^T)
//   dv : k, q, g  backwards (state R)      dk : v, g, q  backwards (state R^T)
// so one kernel computes them all (LinRole).
#include "launch.h"
#include "types16.h"

namespace deer {

constexpr double kLog2e = 1.4426950408889634074;

// log2 of the decay of a step.  Below 2^-256 a decay is zero in float32 whatever it multiplies
// by less than 2^107, and a bounded exponent keeps the differences of sums finite (-inf: a state
// that starts anew).  A NaN stays one.
__device__ __forceinline__ double gate_of(float log_decay) {
    const double g = (double)log_decay * kLog2e;
    return g < -256.0 ? -256.0 : g;
}

// log2 of the factor the walk applies to its state on entering step t: forwards the decay of t,
// backwards that of t + 1; one behind the sequence's end
__device__ __forceinline__ double gate_at(const LinArgs &a, int b, int h, int t, int len, bool rev) {
    const int s = rev ? t + 1 : t;
    if (s >= len) return 0.0;
    return gate_of(a.per_step ? a.log_decay[((size_t)b * a.T + s) * a.H + h] : a.log_decay[h]);
}

__device__ __forceinline__ int length_of(const LinArgs &a, int b) {
    if (!a.lengths) return a.T;
    const int n = a.lengths[b];
    return n < 0 ? 0 : (n > a.T ? a.T : n);
}

template <class Ty>
__device__ __forceinline__ const typename Ty::T *row_of(const LinView &x, int b, int t, int h) {
    return (const typename Ty::T *)x.p + b * x.sb + t * x.st + (h / x.r) * x.sh;
}

// ---- the walk ---------------------------------------------------------------------------------

constexpr int kTile = 64;   // columns of the state per block

int lin_tiles(int Kd, int N) { return (N + kTile - 1) / kTile; }

// One wave per 64 columns of one head's state, which lies in LDS; one step after the other.
template <class Ty>
__global__ __launch_bounds__(64) void k_lin_walk(LinArgs a, LinRole ro) {
    extern __shared__ float lds[];
    float *S = lds;                    // [Kd][64]
    float *qs = S + ro.Kd * kTile, *ks = qs + ro.Kd;
    const int tiles = (ro.N + kTile - 1) / kTile;
    const int tile = blockIdx.x % tiles, bh = blockIdx.x / tiles;
    const int b = bh / a.H, h = bh % a.H, lane = threadIdx.x, n = tile * kTile + lane;
    const bool on = n < ro.N;
    const int len = length_of(a, b);
    const size_t mat = (size_t)ro.Kd * ro.N;
    for (int d = 0; d < ro.Kd; ++d)
        S[d * kTile + lane] = ro.init && on ? ro.init[bh * mat + (size_t)d * ro.init_d + (size_t)n * ro.init_n] : 0.f;
    const int na = (a.T + kLinAnchor - 1) / kLinAnchor;
    for (int i = 0; i < a.T; ++i) {
        const int t = ro.reverse ? a.T - 1 - i : i;
        const bool edge = (t + 1) % kLinAnchor == 0 || t + 1 == a.T;
        float *anc = ro.anchor && edge ? ro.anchor + ((size_t)bh * na + t / kLinAnchor) * mat : nullptr;
        if (anc && ro.reverse && on)
            for (int d = 0; d < ro.Kd; ++d) anc[(size_t)d * ro.N + n] = S[d * kTile + lane];
        float o = 0.f;
        if (t < len) {
            const typename Ty::T *q = row_of<Ty>(ro.q, b, t, h), *k = row_of<Ty>(ro.k, b, t, h);
            for (int d = lane; d < ro.Kd; d += 64) qs[d] = Ty::up(q[d]), ks[d] = Ty::up(k[d]);
            __syncthreads();
            const float g = exp2f((float)gate_at(a, b, h, t, len, ro.reverse));
            const float v = on ? ro.sc_kv * Ty::up(row_of<Ty>(ro.v, b, t, h)[n]) : 0.f;
            for (int d = 0; d < ro.Kd; ++d) {
                const float s = fmaf(ks[d], v, g * S[d * kTile + lane]);
                S[d * kTile + lane] = s;
                o = fmaf(qs[d], s, o);
            }
            o *= ro.sc_o;
            __syncthreads();
        }
        if (on) {
            const size_t at = (((size_t)b * a.T + t) * a.H + h) * ro.N + n;
            if (ro.out_f32) ((float *)ro.out)[at] = o;
            else ((typename Ty::T *)ro.out)[at] = Ty::down(o);
        }
        if (ro.dot) {
            float p = on && t < len ? o * Ty::up(row_of<Ty>(ro.partner, b, t, h)[n]) : 0.f;
            for (int off = 32; off > 0; off >>= 1) p += __shfl_xor(p, off, 64);
            if (lane == 0) ro.dot[((size_t)tile * a.B * a.H + bh) * a.T + t] = p;
        }
        if (anc && !ro.reverse && on)
            for (int d = 0; d < ro.Kd; ++d) anc[(size_t)d * ro.N + n] = S[d * kTile + lane];
    }
    if (ro.fin && on) {
        const float g = ro.reverse ? exp2f((float)gate_at(a, b, h, -1, len, true)) : 1.f;
        for (int d = 0; d < ro.Kd; ++d)
            ro.fin[bh * mat + (size_t)d * ro.fin_d + (size_t)n * ro.fin_n] = g * S[d * kTile + lane];
    }
}

int launch_lin_walk(const LinArgs &a, const LinRole *roles, int nroles, hipStream_t st) {
    return with_dtype(a.dtype, [&](auto ty) {
        using Ty = decltype(ty);
        for (int i = 0; i < nroles; ++i) {
            const LinRole &ro = roles[i];
            const size_t lds = ((size_t)ro.Kd * kTile + 2 * ro.Kd) * sizeof(float);
            DEER_HIP(hipFuncSetAttribute((const void *)k_lin_walk<Ty>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                         (int)lds));
            KTimer kt("k_lin_walk", st);
            hipLaunchKernelGGL(k_lin_walk<Ty>, dim3(a.B * a.H * lin_tiles(ro.Kd, ro.N)), dim3(64), lds, st, a, ro);
            DEER_LAUNCH_CHECK("k_lin_walk");
        }
        return (int)DEER_OK;
    });
}

// ---- the gradient of the log decays --------------------------------------------------------------
//
// dL/dlog a_t = <R_t, a_t S_{t-1}> collects every pair (source j < t, output i >= t).  Over the
// steps t..e-1 before a boundary e, sum_s (q_s dq_s - k_s dk_s) collects those with i < e and takes
// away those with j >= t and i >= e, so with Z_e = <a_e R_e, S_{e-1}> (all pairs across e)
//   dL/dlog a_t = Z_e + sum_{s=t}^{e-1} (q_s dq_s - k_s dk_s).
// Both states are kept every kLinAnchor steps, which bounds the rounding that such a sum gathers.
// One block for each (sequence, head, span of kLinAnchor steps); sums in float64.
constexpr int kSpanThreads = 256, kPer = kLinAnchor / kSpanThreads;

__global__ __launch_bounds__(kSpanThreads) void k_lin_decay_grad(LinArgs a, const float *dq, int q_tiles,
                                                                 const float *dk, int k_tiles, const float *fwd,
                                                                 const float *rev, int elems, double *part,
                                                                 float *out) {
    __shared__ double sh[kSpanThreads];
    const int na = (a.T + kLinAnchor - 1) / kLinAnchor, sp = blockIdx.x % na, bh = blockIdx.x / na;
    const int b = bh / a.H, h = bh % a.H, tid = threadIdx.x, len = length_of(a, b);
    const int t0 = sp * kLinAnchor;
    int t1 = t0 + kLinAnchor;
    t1 = t1 < a.T ? t1 : a.T;
    double z = 0.0;
    const float *S = fwd + ((size_t)bh * na + sp) * elems, *R = rev + ((size_t)bh * na + sp) * elems;
    for (int i = tid; i < elems; i += kSpanThreads) z += (double)S[i] * (double)R[i];
    sh[tid] = z;
    __syncthreads();
    for (int n = kSpanThreads / 2; n > 0; n >>= 1) {
        if (tid < n) sh[tid] += sh[tid + n];
        __syncthreads();
    }
    z = sh[0] * (double)exp2f((float)gate_at(a, b, h, t1 - 1, len, true));
    __syncthreads();
    const size_t plane = (size_t)a.B * a.H * a.T;
    double d[kPer], run = 0.0;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i) {
        const int t = t0 + tid * kPer + i;
        if (t < len) {
            const size_t at = (size_t)bh * a.T + t;
            double x = 0.0;
            for (int n = 0; n < q_tiles; ++n) x += (double)dq[n * plane + at];
            for (int n = 0; n < k_tiles; ++n) x -= (double)dk[n * plane + at];
            run += x;
        }
        d[i] = run;
    }
    sh[tid] = run;
    __syncthreads();
    for (int n = 1; n < kSpanThreads; n <<= 1) {   // sums from this thread to the last
        const double o = tid + n < kSpanThreads ? sh[tid + n] : 0.0;
        __syncthreads();
        sh[tid] += o;
        __syncthreads();
    }
    const double after = z + (tid + 1 < kSpanThreads ? sh[tid + 1] : 0.0);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int t = t0 + tid * kPer + i;
        if (t >= a.T) continue;
        const double v = t < len ? d[i] + after : 0.0;
        if (a.per_step) out[((size_t)b * a.T + t) * a.H + h] = (float)v;
        sum += v;
    }
    if (a.per_step) return;
    __syncthreads();
    sh[tid] = sum;
    __syncthreads();
    for (int n = kSpanThreads / 2; n > 0; n >>= 1) {
        if (tid < n) sh[tid] += sh[tid + n];
        __syncthreads();
    }
    if (tid == 0) part[(size_t)bh * na + sp] = sh[0];
}

// out[h] = sum over sequences and spans of part[b, h, span]
__global__ __launch_bounds__(256) void k_lin_decay_sum(int B, int H, int na, const double *part, float *out) {
    __shared__ double sh[256];
    const int h = blockIdx.x, tid = threadIdx.x;
    double s = 0.0;
    for (long i = tid; i < (long)B * na; i += 256) s += part[((i / na) * H + h) * na + i % na];
    sh[tid] = s;
    __syncthreads();
    for (int n = 128; n > 0; n >>= 1) {
        if (tid < n) sh[tid] += sh[tid + n];
        __syncthreads();
    }
    if (tid == 0) out[h] = (float)sh[0];
}

int launch_lin_decay_grad(const LinArgs &a, const float *dq_dot, int q_tiles, const float *dk_dot, int k_tiles,
                          const float *fwd_anchor, const float *rev_anchor, int elems, double *part, float *dlog_decay,
                          hipStream_t st) {
    const int na = (a.T + kLinAnchor - 1) / kLinAnchor;
    {
        KTimer kt("k_lin_decay_grad", st);
        hipLaunchKernelGGL(k_lin_decay_grad, dim3(a.B * a.H * na), dim3(kSpanThreads), 0, st, a, dq_dot, q_tiles,
                           dk_dot, k_tiles, fwd_anchor, rev_anchor, elems, part, dlog_decay);
        DEER_LAUNCH_CHECK("k_lin_decay_grad");
    }
    if (a.per_step) return DEER_OK;
    KTimer kt("k_lin_decay_sum", st);
    hipLaunchKernelGGL(k_lin_decay_sum, dim3(a.H), dim3(256), 0, st, a.B, a.H, na, part, dlog_decay);
    DEER_LAUNCH_CHECK("k_lin_decay_sum");
    return DEER_OK;
}

// ---- gradients of shared q, k heads ----------------------------------------------------------------

template <class Ty>
__global__ __launch_bounds__(256) void k_lin_head_sum(size_t n, int r, int D, const float *in,
                                                      typename Ty::T *out) {
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
        const size_t row = i / D;
        const float *p = in + row * r * D + i % D;
        float s = 0.f;
        for (int j = 0; j < r; ++j) s += p[(size_t)j * D];
        out[i] = Ty::down(s);
    }
}

int launch_lin_head_sum(int dtype, size_t rows, int Hk, int r, int D, const float *in, void *out, hipStream_t st) {
    const size_t n = rows * Hk * D, blocks = (n + 255) / 256;
    return with_dtype(dtype, [&](auto ty) {
        using Ty = decltype(ty);
        KTimer kt("k_lin_head_sum", st);
        hipLaunchKernelGGL(k_lin_head_sum<Ty>, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, st, n, r,
                           D, in, (typename Ty::T *)out);
        DEER_LAUNCH_CHECK("k_lin_head_sum");
        return (int)DEER_OK;
    });
}

// ---- one step ----------------------------------------------------------------------------------------

// One block per 64 columns of one head's state; a thread owns one column of every 4th row.
template <class Ty>
__global__ __launch_bounds__(256) void k_lin_step(LinStep a) {
    __shared__ float qs[256], ks[256], red[4][64];
    const int tiles = (a.Dv + 63) / 64, tile = blockIdx.x % tiles, bh = blockIdx.x / tiles;
    const int b = bh / a.H, h = bh % a.H, c = threadIdx.x & 63, w = threadIdx.x >> 6, n = tile * 64 + c;
    const bool on = n < a.Dv;
    typename Ty::T *o = (typename Ty::T *)a.o + (size_t)bh * a.Dv + n;
    if (a.lengths && a.lengths[b] <= 0) {
        if (w == 0 && on) *o = Ty::down(0.f);
        return;
    }
    const typename Ty::T *q = row_of<Ty>(a.q, b, 0, h), *k = row_of<Ty>(a.k, b, 0, h);
    for (int d = threadIdx.x; d < a.Dk; d += 256) qs[d] = Ty::up(q[d]), ks[d] = Ty::up(k[d]);
    __syncthreads();
    const float g = exp2f((float)gate_of(a.log_decay[a.per_seq ? (size_t)bh : h]));
    float acc = 0.f;
    if (on) {
        const float v = Ty::up(row_of<Ty>(a.v, b, 0, h)[n]);
        float *S = a.state + (size_t)bh * a.Dk * a.Dv + n;
        for (int d = w; d < a.Dk; d += 4) {
            const float s = fmaf(ks[d], v, g * S[(size_t)d * a.Dv]);
            S[(size_t)d * a.Dv] = s;
            acc = fmaf(qs[d], s, acc);
        }
    }
    red[w][c] = acc;
    __syncthreads();
    if (w == 0 && on) *o = Ty::down(a.scale * ((red[0][c] + red[1][c]) + (red[2][c] + red[3][c])));
}

int launch_lin_step(const LinStep &a, hipStream_t st) {
    return with_dtype(a.dtype, [&](auto ty) {
        using Ty = decltype(ty);
        KTimer kt("k_lin_step", st);
        hipLaunchKernelGGL(k_lin_step<Ty>, dim3(a.B * a.H * ((a.Dv + 63) / 64)), dim3(256), 0, st, a);
        DEER_LAUNCH_CHECK("k_lin_step");
        return (int)DEER_OK;
    });
}

}  // namespace deer
