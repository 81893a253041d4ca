// Layer normalisation, forward and adjoint (deer_layernorm, deer_layernorm_adjoint).
#include "launch.h"
#include "types16.h"

namespace deer {

constexpr int kRowThreads = 256;

// sum over the block, the same order every time
__device__ __forceinline__ float block_sum(float v, float *sh) {
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

// One block per row.  The variance is the mean of the squared differences from the mean, not a
// difference of two large sums.
template <class Ty, class Wt>
__global__ __launch_bounds__(kRowThreads) void k_layernorm(NormArgs a, typename Ty::T *y, float *mean, float *rstd) {
    __shared__ float sh[4];
    const typename Wt::T *w = (const typename Wt::T *)a.w, *bb = (const typename Wt::T *)a.b;
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const typename Ty::T *x = (const typename Ty::T *)a.x + row * a.D;
        const size_t wr = (row % a.G) * a.D;
        float s = 0.f;
        for (int i = threadIdx.x; i < a.D; i += kRowThreads) s += Ty::up(x[i]);
        const float m = block_sum(s, sh) / (float)a.D;
        s = 0.f;
        for (int i = threadIdx.x; i < a.D; i += kRowThreads) {
            const float d = Ty::up(x[i]) - m;
            s = fmaf(d, d, s);
        }
        const float r = 1.f / sqrtf(block_sum(s, sh) / (float)a.D + a.eps);
        for (int i = threadIdx.x; i < a.D; i += kRowThreads) {
            float v = (Ty::up(x[i]) - m) * r;
            if (w) v *= Wt::up(w[wr + i]);
            if (bb) v += Wt::up(bb[wr + i]);
            y[row * a.D + i] = Ty::down(v);
        }
        if (threadIdx.x == 0) {
            if (mean) mean[row] = m;
            if (rstd) rstd[row] = r;
        }
    }
}

template <class Ty, class Wt>
__global__ __launch_bounds__(kRowThreads) void k_layernorm_dx(NormArgs a, const typename Ty::T *g, const float *mean,
                                                              const float *rstd, typename Ty::T *dx) {
    __shared__ float sh[4];
    const typename Wt::T *w = (const typename Wt::T *)a.w;
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const typename Ty::T *x = (const typename Ty::T *)a.x + row * a.D, *gr = g + row * a.D;
        const size_t wr = (row % a.G) * a.D;
        const float m = mean[row], r = rstd[row];
        float s1 = 0.f, s2 = 0.f;
        for (int i = threadIdx.x; i < a.D; i += kRowThreads) {
            const float u = Ty::up(gr[i]) * (w ? Wt::up(w[wr + i]) : 1.f), xh = (Ty::up(x[i]) - m) * r;
            s1 += u;
            s2 = fmaf(u, xh, s2);
        }
        s1 = block_sum(s1, sh) / (float)a.D;
        s2 = block_sum(s2, sh) / (float)a.D;
        for (int i = threadIdx.x; i < a.D; i += kRowThreads) {
            const float u = Ty::up(gr[i]) * (w ? Wt::up(w[wr + i]) : 1.f), xh = (Ty::up(x[i]) - m) * r;
            dx[row * a.D + i] = Ty::down(r * (u - s1 - xh * s2));
        }
    }
}

constexpr int kSplits = 64;   // partial sums over the rows

// partial sums of split blockIdx.y (rows group + G i, i = split, split + kSplits, ...)
template <class Ty>
__global__ __launch_bounds__(256) void k_layernorm_dw_part(NormArgs a, const typename Ty::T *g, const float *mean,
                                                           const float *rstd, float *part) {
    const int n = a.G * a.D, i = blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int grp = i / a.D, c = i % a.D;
    float sw = 0.f, sb = 0.f;
    for (size_t row = grp + (size_t)a.G * blockIdx.y; row < a.rows; row += (size_t)a.G * kSplits) {
        const float gv = Ty::up(g[row * a.D + c]);
        sw = fmaf(gv, (Ty::up(((const typename Ty::T *)a.x)[row * a.D + c]) - mean[row]) * rstd[row], sw);
        sb += gv;
    }
    part[((size_t)blockIdx.y * 2) * n + i] = sw;
    part[((size_t)blockIdx.y * 2 + 1) * n + i] = sb;
}

__global__ __launch_bounds__(256) void k_layernorm_dw_sum(int n, const float *part, float *dw, float *db) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    double sw = 0.0, sb = 0.0;
    for (int s = 0; s < kSplits; ++s) sw += part[((size_t)s * 2) * n + i], sb += part[((size_t)s * 2 + 1) * n + i];
    if (dw) dw[i] = (float)sw;
    if (db) db[i] = (float)sb;
}

template <class Fn>
static int with_types(int dtype, int wtype, Fn f) {
    return with_dtype(dtype, [&](auto ty) {
        if (wtype == DEER_F32) return f(ty, F32{});
        return f(ty, ty);
    });
}

int launch_layernorm(const NormArgs &a, void *y, float *mean, float *rstd, hipStream_t st) {
    return with_types(a.dtype, a.wtype, [&](auto ty, auto wt) {
        using Ty = decltype(ty);
        using Wt = decltype(wt);
        KTimer kt("k_layernorm", st);
        hipLaunchKernelGGL((k_layernorm<Ty, Wt>), dim3((unsigned)(a.rows < 65536 ? a.rows : 65536)), dim3(kRowThreads), 0,
                           st, a, (typename Ty::T *)y, mean, rstd);
        DEER_LAUNCH_CHECK("k_layernorm");
        return (int)DEER_OK;
    });
}

size_t layernorm_adjoint_ws_bytes(size_t rows, int G, int D) { return (size_t)kSplits * 2 * G * D * sizeof(float); }

int launch_layernorm_adjoint(const NormArgs &a, const void *g, const float *mean, const float *rstd, void *dx,
                             float *dw, float *db, void *ws, hipStream_t st) {
    return with_types(a.dtype, a.wtype, [&](auto ty, auto wt) {
        using Ty = decltype(ty);
        using Wt = decltype(wt);
        using T = typename Ty::T;
        if (dx) {
            KTimer kt("k_layernorm_dx", st);
            hipLaunchKernelGGL((k_layernorm_dx<Ty, Wt>), dim3((unsigned)(a.rows < 65536 ? a.rows : 65536)),
                               dim3(kRowThreads), 0, st, a, (const T *)g, mean, rstd, (T *)dx);
            DEER_LAUNCH_CHECK("k_layernorm_dx");
        }
        if (!dw && !db) return (int)DEER_OK;
        const int n = a.G * a.D, blocks = (n + 255) / 256;
        {
            KTimer kt("k_layernorm_dw_part", st);
            hipLaunchKernelGGL(k_layernorm_dw_part<Ty>, dim3(blocks, kSplits), dim3(256), 0, st, a, (const T *)g, mean,
                               rstd, (float *)ws);
            DEER_LAUNCH_CHECK("k_layernorm_dw_part");
        }
        KTimer kt("k_layernorm_dw_sum", st);
        hipLaunchKernelGGL(k_layernorm_dw_sum, dim3(blocks), dim3(256), 0, st, n, (const float *)ws, dw, db);
        DEER_LAUNCH_CHECK("k_layernorm_dw_sum");
        return (int)DEER_OK;
    });
}

}  // namespace deer
