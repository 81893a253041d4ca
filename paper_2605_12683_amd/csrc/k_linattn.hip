// Linear attention with a decay for each head (deer_linattn, deer_linattn_adjoint,
// deer_linattn_step).
//
// The recurrence S_t = a_t S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t and its three large gradients
// are the same walk with the operands in other places:
//   o  : q, k, v  forwards                 dq : g, v, k  forwards (the state is S^T)
//   dv : k, q, g  backwards (state R)      dk : v, g, q  backwards (state R^T)
// so one kernel computes them all (LinRole).
#include "linwalk.h"

namespace deer {

// ---- walks in segments ----------------------------------------------------------------------------
//
// With few heads the walks alone do not fill the chip, so a sequence is cut into segments: a first
// walk finds the state that each but the last adds by itself, and the walks proper start all at once
// from the states entering the segments.  Few segments are added up by the walks' blocks themselves;
// with more, k_lin_join turns what each adds into what enters it (one pass over the segments, in
// place).  That reads k and v twice.

// four elements of one head's state per thread, the segments in the walk's order, eight of them
// loaded at a time (32 heads of 128 x 128, 16 segments: 62 MiB in 12 us)
__global__ __launch_bounds__(256) void k_lin_join(LinArgs a, LinRoles rs) {
    const LinRole &ro = rs.r[blockIdx.y];
    const int mat = ro.Kd * ro.N, per = (mat + 1023) / 1024;
    const int bh = blockIdx.x / per, e = (blockIdx.x % per * 256 + threadIdx.x) * 4;
    if (bh >= a.B * a.H || e >= mat) return;
    const int left = mat - e < 4 ? mat - e : 4;
    const bool four = mat % 4 == 0;
    float S[4] = {0.f, 0.f, 0.f, 0.f};
    if (ro.init)
        for (int r = 0; r < left; ++r) {
            const int d = (e + r) / ro.N, n = (e + r) % ro.N;
            S[r] = ro.init[(size_t)bh * mat + (size_t)d * ro.init_d + (size_t)n * ro.init_n];
        }
    float *seg = ro.seg + (size_t)bh * a.nseg * mat + e;
    const SegDecay *dec = ro.seg_decay + (size_t)bh * a.nseg;
    constexpr int U = 8;
    for (int i0 = 0; i0 < a.nseg; i0 += U) {
        float x[U][4];
        SegDecay f[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u, s = ro.reverse ? a.nseg - 1 - i : i;
            const bool on = i < a.nseg - 1;
            const float *p = seg + (size_t)s * mat;
            v4f y = {0.f, 0.f, 0.f, 0.f};
            if (on && four) y = *(const v4f *)p;
#pragma unroll
            for (int r = 0; r < 4; ++r) x[u][r] = y[r];
            if (on && !four)
                for (int r = 0; r < left; ++r) x[u][r] = p[r];
            f[u] = on ? dec[s] : SegDecay{0.f, 0};
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u, s = ro.reverse ? a.nseg - 1 - i : i;
            if (i >= a.nseg) break;
            float *p = seg + (size_t)s * mat;
            if (four) *(v4f *)p = v4f{S[0], S[1], S[2], S[3]};
            else
                for (int r = 0; r < left; ++r) p[r] = S[r];
#pragma unroll
            for (int r = 0; r < 4; ++r) S[r] = decayed(f[u], S[r], x[u][r]);
        }
    }
}

int launch_lin_join(const LinArgs &a, const LinRole *roles, int nroles, hipStream_t st) {
    LinRoles rs{};
    int most = 0;
    for (int i = 0; i < nroles; ++i) {
        rs.r[i] = roles[i];
        const int n = (roles[i].Kd * roles[i].N + 1023) / 1024;
        most = n > most ? n : most;
    }
    KTimer kt("k_lin_join", st);
    hipLaunchKernelGGL(k_lin_join, dim3((unsigned)(a.B * a.H * most), nroles), dim3(256), 0, st, a, rs);
    DEER_LAUNCH_CHECK("k_lin_join");
    return DEER_OK;
}

int lin_tiles(int Kd, int N) {
    const int nb = nb_of(kt_of(Kd), N);
    return (N + nb - 1) / nb;
}

int lin_resident(int dtype, int Kd, int N, bool dots) {
    return with_dtype(dtype, [&](auto ty) {
        constexpr int NPI = InParts<decltype(ty)>::n;
        return with_walk_shape<NPI>(Kd, N, false, [&](auto s) {
            return dots ? LinTile<NPI, s.KT, s.NW, s.CT, kOutDots>::waves * 4 / s.NW
                        : LinTile<NPI, s.KT, s.NW, s.CT, kOut>::waves * 4 / s.NW;
        });
    });
}

bool lin_same_tile(int Kd, int N, int Kd2, int N2) {
    return kt_of(Kd) == kt_of(Kd2) && nb_of(kt_of(Kd), N) == nb_of(kt_of(Kd2), N2);
}

int launch_lin_walk(const LinArgs &a, const LinRole *roles, int nroles, bool states, bool dots, hipStream_t st) {
    if (a.dtype == DEER_F32) return launch_lin_walk_f32(a, roles, nroles, states, dots, st);
    if (a.dtype == DEER_BF16) return launch_lin_walk_bf16(a, roles, nroles, states, dots, st);
    return launch_lin_walk_f16(a, roles, nroles, states, dots, st);
}

// ---- the gradient of the log decays --------------------------------------------------------------
//
// dL/dlog a_t = <R_t, a_t S_{t-1}> collects every pair (source j < t, output i >= t).  Over the
// steps t..e-1 before a boundary e, sum_s (q_s dq_s - k_s dk_s) collects those with i < e and takes
// away those with j >= t and i >= e, so with Z_e = <a_e R_e, S_{e-1}> (all pairs across e)
//   dL/dlog a_t = Z_e + sum_{s=t}^{e-1} (q_s dq_s - k_s dk_s).
// Both states are kept every kLinAnchor steps, which bounds the rounding that such a sum gathers.
// One block for each (sequence, head, span of kLinAnchor steps), bound by reading the states (64 heads
// of 128 x 128, 4096 steps: 32 MiB of states in 14 us); sums in float64.
constexpr int kSpanThreads = 256, kPer = kLinAnchor / kSpanThreads;

__global__ __launch_bounds__(kSpanThreads) void k_lin_decay_grad(LinArgs a, const float *dq, int q_tiles,
                                                                 const float *dk, int k_tiles, const float *fwd,
                                                                 const float *rev, int elems, bool from_zero,
                                                                 double *part, float *out) {
    __shared__ double sh[kSpanThreads];
    const int na = (a.T + kLinAnchor - 1) / kLinAnchor, sp = blockIdx.x % na, bh = blockIdx.x / na;
    const int b = bh / a.H, h = bh % a.H, tid = threadIdx.x, len = length_of(a, b);
    const int t0 = sp * kLinAnchor;
    int t1 = t0 + kLinAnchor;
    t1 = t1 < a.T ? t1 : a.T;
    double z = 0.0;
    const float *S = fwd + ((size_t)bh * na + sp) * elems, *R = rev + ((size_t)bh * na + sp) * elems;
    if (elems % 4 == 0) {
        const v4f *S4 = (const v4f *)S, *R4 = (const v4f *)R;
#pragma unroll 8
        for (int i = tid; i < elems / 4; i += kSpanThreads) {
            const v4f s = S4[i], r = R4[i];
            z += ((double)s[0] * r[0] + (double)s[1] * r[1]) + ((double)s[2] * r[2] + (double)s[3] * r[3]);
        }
    } else {
        for (int i = tid; i < elems; i += kSpanThreads) z += (double)S[i] * (double)R[i];
    }
    sh[tid] = z;
    __syncthreads();
    for (int n = kSpanThreads / 2; n > 0; n >>= 1) {
        if (tid < n) sh[tid] += sh[tid + n];
        __syncthreads();
    }
    z = sh[0] * (double)__builtin_amdgcn_exp2f((float)gate_of(gate_raw(a, b, h, t1 - 1, len, true)));
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
        // nothing to decay in the first step from no state, nothing left of it by a decay of zero: exactly 0
        const bool none = t >= len || (from_zero && t == 0) || gate_of(gate_raw(a, b, h, t, len, false)) == -256.0;
        const double v = none ? 0.0 : d[i] + after;
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
                          const float *fwd_anchor, const float *rev_anchor, int elems, bool from_zero, double *part,
                          float *dlog_decay, hipStream_t st) {
    const int na = (a.T + kLinAnchor - 1) / kLinAnchor;
    {
        KTimer kt("k_lin_decay_grad", st);
        hipLaunchKernelGGL(k_lin_decay_grad, dim3(a.B * a.H * na), dim3(kSpanThreads), 0, st, a, dq_dot, q_tiles,
                           dk_dot, k_tiles, fwd_anchor, rev_anchor, elems, from_zero, part, dlog_decay);
        DEER_LAUNCH_CHECK("k_lin_decay_grad");
    }
    if (a.per_step) return DEER_OK;
    KTimer kt("k_lin_decay_sum", st);
    hipLaunchKernelGGL(k_lin_decay_sum, dim3(a.H), dim3(256), 0, st, a.B, a.H, na, part, dlog_decay);
    DEER_LAUNCH_CHECK("k_lin_decay_sum");
    return DEER_OK;
}

// ---- gradients of shared q, k heads ----------------------------------------------------------------
//
// Each head's walk leaves its dq and dk in float32, and their sums are rounded once; bound by memory
// where the sequences are long (7 us, most of it the launch's own, for 3 x 2500 steps of 6 heads of 48).

// dq (blockIdx.y 0) and dk (1)
template <class Ty>
__global__ __launch_bounds__(256) void k_lin_head_sum(size_t n, int r, uint32_t D, const float *dq, const float *dk,
                                                      typename Ty::T *dq_out, typename Ty::T *dk_out) {
    const float *in = blockIdx.y ? dk : dq;
    typename Ty::T *out = blockIdx.y ? dk_out : dq_out;
    for (size_t i0 = (size_t)blockIdx.x * 256; i0 < n; i0 += (size_t)gridDim.x * 256) {
        if (i0 + threadIdx.x >= n) return;
        // (one long division for all threads)
        const size_t row0 = i0 / D;
        const uint32_t d0 = (uint32_t)(i0 - row0 * D) + threadIdx.x, row = d0 / D, d = d0 % D;
        const float *p = in + (row0 + row) * r * D + d;
        float s = 0.f;
        for (int j = 0; j < r; ++j) s += p[(size_t)j * D];
        out[i0 + threadIdx.x] = Ty::down(s);
    }
}

int launch_lin_head_sum(int dtype, size_t rows, int Hk, int r, int D, const float *dq, const float *dk, void *dq_out,
                        void *dk_out, hipStream_t st) {
    const size_t n = rows * Hk * D, blocks = (n + 255) / 256;
    return with_dtype(dtype, [&](auto ty) {
        using Ty = decltype(ty);
        KTimer kt("k_lin_head_sum", st);
        hipLaunchKernelGGL(k_lin_head_sum<Ty>, dim3((unsigned)(blocks < 65536 ? blocks : 65536), 2), dim3(256), 0, st, n, r,
                           (uint32_t)D, dq, dk, (typename Ty::T *)dq_out, (typename Ty::T *)dk_out);
        DEER_LAUNCH_CHECK("k_lin_head_sum");
        return (int)DEER_OK;
    });
}

// ---- one step ----------------------------------------------------------------------------------------

template <class Ty>
__device__ __forceinline__ const typename Ty::T *row_of(const LinView &x, int b, int h) {
    return (const typename Ty::T *)x.p + b * x.sb + (h / x.r) * x.sh;
}

// One block per 64 columns of one head's state, which is read and written once: memory bounds a batch
// (256 sequences, 32 heads of 128 x 128: 1.08 GB in 210 us, 5.1 TB/s), latency a single sequence.  A thread owns W
// columns of every (4 W)th row, up to eight rows loaded before the first is used; W = 4 where Dv and
// the state's address allow loads of 16 bytes.
template <class Ty, int W>
__global__ __launch_bounds__(256) void k_lin_step(LinStep a) {
    constexpr int LC = 64 / W, RG = 256 / LC, U = 8;   // lanes per row, rows at a time, rows in flight
    __shared__ float qs[256], ks[256], red[RG][64];
    const int tiles = (a.Dv + 63) / 64, tile = blockIdx.x % tiles, bh = blockIdx.x / tiles;
    const int b = bh / a.H, h = bh % a.H, cl = threadIdx.x % LC, rg = threadIdx.x / LC, n = tile * 64 + cl * W;
    const bool on = n < a.Dv;
    typename Ty::T *o = (typename Ty::T *)a.o + (size_t)bh * a.Dv + tile * 64;
    if (a.lengths && a.lengths[b] <= 0) {
        if (threadIdx.x < 64 && tile * 64 + (int)threadIdx.x < a.Dv) o[threadIdx.x] = Ty::down(0.f);
        return;
    }
    typedef float vf __attribute__((ext_vector_type(W)));
    vf *S = (vf *)(a.state + (size_t)bh * a.Dk * a.Dv + n);
    const size_t row = a.Dv / W;                       // in vf
    vf s[U];
    auto load = [&](int d0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (on && d0 + u * RG < a.Dk) s[u] = S[(size_t)(d0 + u * RG) * row];
    };
    load(rg);
    const typename Ty::T *q = row_of<Ty>(a.q, b, h), *k = row_of<Ty>(a.k, b, h);
    for (int d = threadIdx.x; d < a.Dk; d += 256) qs[d] = Ty::up(q[d]), ks[d] = Ty::up(k[d]);
    const float g = __builtin_amdgcn_exp2f((float)gate_of(a.log_decay[a.per_seq ? (size_t)bh : h]));
    vf v = {}, acc = {};
    if (on)
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = Ty::up(row_of<Ty>(a.v, b, h)[n + i]);
    lds_barrier();
    for (int d0 = rg; d0 < a.Dk; d0 += U * RG) {
        if (d0 != rg) load(d0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int d = d0 + u * RG;
            if (!on || d >= a.Dk) continue;
            const float kd = ks[d], qd = qs[d];
#pragma unroll
            for (int i = 0; i < W; ++i) {
                s[u][i] = fmaf(kd, v[i], g * s[u][i]);
                acc[i] = fmaf(qd, s[u][i], acc[i]);
            }
            S[(size_t)d * row] = s[u];
        }
    }
#pragma unroll
    for (int i = 0; i < W; ++i) red[rg][cl * W + i] = acc[i];
    lds_barrier();
    if (threadIdx.x < 64 && tile * 64 + (int)threadIdx.x < a.Dv) {
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < RG; ++i) x += red[i][threadIdx.x];
        o[threadIdx.x] = Ty::down(a.scale * x);
    }
}

int launch_lin_step(const LinStep &a, hipStream_t st) {
    return with_dtype(a.dtype, [&](auto ty) {
        using Ty = decltype(ty);
        KTimer kt("k_lin_step", st);
        const dim3 grid(a.B * a.H * ((a.Dv + 63) / 64));
        if (a.Dv % 4 == 0 && ((uintptr_t)a.state & 15) == 0)
            hipLaunchKernelGGL((k_lin_step<Ty, 4>), grid, dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((k_lin_step<Ty, 1>), grid, dim3(256), 0, st, a);
        DEER_LAUNCH_CHECK("k_lin_step");
        return (int)DEER_OK;
    });
}

}  // namespace deer
