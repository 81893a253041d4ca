// Layer normalisation, forward and adjoint (deer_layernorm, deer_layernorm_adjoint).
//
// Both directions read each row once and write it once and do a few operations per element, so
// memory bounds them (in bf16, 32768 rows: of 2048 forwards 54 us, 5.0 TB/s; of 4096 backwards 157 us,
// 5.1 TB/s, and 5 us for the partial sums).  A team of TEAM threads holds a whole row in registers (NV
// units of 16 bytes a thread) and takes every NT-th row, loading the next one while it reduces this
// one; NT is a multiple of G, so that a team's rows share their weights, which it keeps in registers
// too.  The adjoint adds its rows' part of dw and db in registers and writes one partial sum per block
// (G = 1) or team, which k_layernorm_sum adds up in float64: no atomics, the same order every time.
//
// Rows of more than 16384 elements, a team's most, are read once for every sum instead.
#include <type_traits>

#include "launch.h"
#include "types16.h"

namespace deer {

// v plus that of the lane whose number differs in the bit OFF alone, with no trip through LDS.  Within
// 16 lanes by rotation: lanes 8 apart are the same both ways, and of numbers that repeat every
// 2 OFF lanes those OFF apart are.
template <int OFF>
__device__ __forceinline__ float add_across(float v) {
    const uint32_t u = __float_as_uint(v);
    if constexpr (OFF == 32) {
        const auto p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        return __uint_as_float(p[0]) + __uint_as_float(p[1]);
    } else if constexpr (OFF == 16) {
        const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        return __uint_as_float(p[0]) + __uint_as_float(p[1]);
    } else {
        return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, 0x120 + OFF, 15, 15, false));   // row_ror
    }
}

// sum over a team; all its threads get it, the terms are always added in the same order
template <int TEAM>
struct TeamSum {
    float *sh;        // 2 * TEAM / 64 floats, TEAM > 64 (one team per block)
    int flip = 0;

    __device__ __forceinline__ float operator()(float v) {
        if constexpr (TEAM >= 64) v = add_across<16>(add_across<32>(v));
        v = add_across<1>(add_across<2>(add_across<4>(add_across<8>(v))));
        if constexpr (TEAM > 64) {
            constexpr int W = TEAM / 64;
            float *s = sh + flip * W;   // two buffers: one barrier a sum
            flip ^= 1;
            if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
            lds_barrier();
            v = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) v += s[i];
        }
        return v;
    }
};

__device__ __forceinline__ float weight_at(const NormArgs &a, const void *w, size_t i, float none) {
    if (!w) return none;
    if (a.wtype == DEER_F32) return ((const float *)w)[i];
    if (a.wtype == DEER_BF16) return (float)((const __bf16 *)w)[i];
    return (float)((const _Float16 *)w)[i];
}

template <int E, int NV, int TEAM>
__device__ __forceinline__ void load_weights(const NormArgs &a, const void *w, int group, int lane, float none,
                                             float (&out)[NV][E]) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int d = (v * TEAM + lane) * E + e;
            out[v][e] = d < a.D ? weight_at(a, w, (size_t)group * a.D + d, none) : 0.f;
        }
}

constexpr int block_of(int team) { return team <= 64 ? 256 : team; }   // a team of several waves has its block to itself

template <class Ty, int TEAM, int NV>
__global__ __launch_bounds__(block_of(TEAM)) void k_layernorm(NormArgs a, int nt, bool vec, typename Ty::T *y,
                                                              float *mean, float *rstd) {
    using T = typename Ty::T;
    constexpr int E = 16 / sizeof(T), TPB = block_of(TEAM) / TEAM;
    __shared__ float sh[TEAM > 64 ? 2 * TEAM / 64 : 1];
    TeamSum<TEAM> sum{sh};
    const int lane = threadIdx.x % TEAM, team = blockIdx.x * TPB + threadIdx.x / TEAM;
    if (team >= nt) return;   // whole teams; none of more than a wave
    const T *x = (const T *)a.x;
    float w[NV][E], b[NV][E];
    v4u next[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) next[v] = load_unit<Ty>(x + (size_t)team * a.D, (v * TEAM + lane) * E, a.D, vec);
    load_weights<E, NV, TEAM>(a, a.w, team % a.G, lane, 1.f, w);
    load_weights<E, NV, TEAM>(a, a.b, team % a.G, lane, 0.f, b);
    const float width = (float)a.D;   // divided by: the mean of equal numbers is that number
    for (size_t row = team; row < a.rows; row += nt) {
        float f[NV][E], s = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            unpack_unit<Ty>(next[v], f[v]);
#pragma unroll
            for (int e = 0; e < E; ++e) s += f[v][e];
        }
        if (row + nt < a.rows)
#pragma unroll
            for (int v = 0; v < NV; ++v) next[v] = load_unit<Ty>(x + (row + nt) * a.D, (v * TEAM + lane) * E, a.D, vec);
        const float m = sum(s) / width;
        s = 0.f;
        // the variance as the mean of squared differences, not a difference of two large sums
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                f[v][e] -= m;
                if ((v * TEAM + lane) * E + e < a.D) s = fmaf(f[v][e], f[v][e], s);
            }
        const float r = 1.f / sqrtf(sum(s) / width + a.eps);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float o[E];
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = fmaf(f[v][e] * r, w[v][e], b[v][e]);
            store_unit<Ty>(y + row * a.D, (v * TEAM + lane) * E, a.D, vec, o);
        }
        if (lane == 0) {
            if (mean) mean[row] = m;
            if (rstd) rstd[row] = r;
        }
    }
}

// part: [partials][2][D] (dw, db), one partial per block with G = 1, else per team; null: dx only
template <class Ty, int TEAM, int NV>
__global__ __launch_bounds__(block_of(TEAM)) void k_layernorm_adj(NormArgs a, int nt, bool vec, const typename Ty::T *g,
                                                                  const float *mean, const float *rstd,
                                                                  typename Ty::T *dx, float *part) {
    using T = typename Ty::T;
    constexpr int E = 16 / sizeof(T), TPB = block_of(TEAM) / TEAM;
    __shared__ float sh[TEAM > 64 ? 2 * TEAM / 64 : 1];
    __shared__ float cols[TPB > 1 ? 2 * TEAM * NV * E : 1];
    TeamSum<TEAM> sum{sh};
    const int lane = threadIdx.x % TEAM, in_block = threadIdx.x / TEAM, team = blockIdx.x * TPB + in_block;
    const T *x = (const T *)a.x;
    const bool on = team < nt;
    // of the next row, x and g are loaded while this one is reduced, or where registers are few only x, or
    // none (1024 threads, 128 registers each)
    constexpr bool BOTH = TEAM * NV < 2048, AHEAD = TEAM < 1024;
    float dw[NV][E], db[NV][E];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < E; ++e) dw[v][e] = db[v][e] = 0.f;
    if (on) {
        float w[NV][E];
        v4u nx[NV], ng[NV];
        float nm, nr;
        auto load_x = [&](size_t row) {
#pragma unroll
            for (int v = 0; v < NV; ++v) nx[v] = load_unit<Ty>(x + row * a.D, (v * TEAM + lane) * E, a.D, vec);
            nm = mean[row], nr = rstd[row];
        };
        auto load_g = [&](size_t row) {
#pragma unroll
            for (int v = 0; v < NV; ++v) ng[v] = load_unit<Ty>(g + row * a.D, (v * TEAM + lane) * E, a.D, vec);
        };
        if (AHEAD) load_x(team);
        if (BOTH) load_g(team);
        load_weights<E, NV, TEAM>(a, a.w, team % a.G, lane, 1.f, w);
        const float width = (float)a.D;   // divided by: the mean of equal numbers is that number
        for (size_t row = team; row < a.rows; row += nt) {
            if (!AHEAD) load_x(row);
            if (!BOTH) load_g(row);
            const float m = nm, r = nr;
            float xh[NV][E], u[NV][E], s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                unpack_unit<Ty>(nx[v], xh[v]);
                unpack_unit<Ty>(ng[v], u[v]);
#pragma unroll
                for (int e = 0; e < E; ++e) {   // g is zero beyond D, xh then counts for nothing
                    xh[v][e] = (xh[v][e] - m) * r;
                    dw[v][e] = fmaf(u[v][e], xh[v][e], dw[v][e]);
                    db[v][e] += u[v][e];
                    u[v][e] *= w[v][e];
                    s1 += u[v][e];
                    s2 = fmaf(u[v][e], xh[v][e], s2);
                }
            }
            if (AHEAD && row + nt < a.rows) {
                load_x(row + nt);
                if (BOTH) load_g(row + nt);
            }
            if (!dx) continue;
            s1 = sum(s1) / width;
            s2 = sum(s2) / width;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float o[E];
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = r * (u[v][e] - s1 - xh[v][e] * s2);
                store_unit<Ty>(dx + row * a.D, (v * TEAM + lane) * E, a.D, vec, o);
            }
        }
    }
    if (!part) return;
    if (TPB == 1 || a.G > 1) {
        if (!on) return;
        float *p = part + (size_t)team * 2 * a.D;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int d = (v * TEAM + lane) * E + e;
                if (d < a.D) p[d] = dw[v][e], p[a.D + d] = db[v][e];
            }
        return;
    }
    // the block's teams, one after the other
    for (int i = 0; i < TPB; ++i) {
        if (in_block == i)
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int d = (v * TEAM + lane) * E + e, n = TEAM * NV * E;
                    cols[d] = (i ? cols[d] : 0.f) + dw[v][e];
                    cols[n + d] = (i ? cols[n + d] : 0.f) + db[v][e];
                }
        __syncthreads();
    }
    float *p = part + (size_t)blockIdx.x * 2 * a.D;
    for (int d = threadIdx.x; d < a.D; d += block_of(TEAM)) {
        p[d] = cols[d];
        p[a.D + d] = cols[TEAM * NV * E + d];
    }
}

// out[g, d] = sum over the partials of group g (g, g + G, ...): 32 columns by SL slices a block, in
// float64.  Each slice's chain of loads is what takes the time: 32 slices where a group has hundreds
// of partials (515 columns of 701: 9.2 us with 8 slices, 6.1 with 32), 8 where it has few.
template <int SL>
__global__ __launch_bounds__(32 * SL) void k_layernorm_sum(int G, int D, int np, const float *part, float *dw,
                                                           float *db) {
    __shared__ double sh[SL][32];
    float *out = blockIdx.y ? db : dw;
    if (!out) return;
    const int per = (D + 31) / 32, grp = blockIdx.x / per, c = threadIdx.x & 31, sl = threadIdx.x >> 5;
    const int d = blockIdx.x % per * 32 + c;
    double s = 0.0;
    if (d < D) {
        const float *p = part + (size_t)blockIdx.y * D + d;
        const size_t step = (size_t)2 * D;
#pragma unroll 8
        for (int i = grp + G * sl; i < np; i += SL * G) s += (double)p[i * step];
    }
    sh[sl][c] = s;
    __syncthreads();
    if (sl == 0 && d < D) {
        for (int i = 1; i < SL; ++i) s += sh[i][c];
        out[(size_t)grp * D + d] = (float)s;
    }
}

// ---- rows beyond the registers ------------------------------------------------------------------

constexpr int kLongThreads = 1024, kLongSplits = 64;

template <class Ty>
__global__ __launch_bounds__(kLongThreads) void k_layernorm_long(NormArgs a, typename Ty::T *y, float *mean,
                                                                 float *rstd) {
    __shared__ float sh[2 * kLongThreads / 64];
    TeamSum<kLongThreads> sum{sh};
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const typename Ty::T *x = (const typename Ty::T *)a.x + row * a.D;
        const size_t wr = (row % a.G) * a.D;
        float s = 0.f;
        for (int i = threadIdx.x; i < a.D; i += kLongThreads) s += Ty::up(x[i]);
        const float m = sum(s) / (float)a.D;
        s = 0.f;
        for (int i = threadIdx.x; i < a.D; i += kLongThreads) {
            const float d = Ty::up(x[i]) - m;
            s = fmaf(d, d, s);
        }
        const float r = 1.f / sqrtf(sum(s) / (float)a.D + a.eps);
        for (int i = threadIdx.x; i < a.D; i += kLongThreads)
            y[row * a.D + i] =
                Ty::down(fmaf((Ty::up(x[i]) - m) * r, weight_at(a, a.w, wr + i, 1.f), weight_at(a, a.b, wr + i, 0.f)));
        if (threadIdx.x == 0) {
            if (mean) mean[row] = m;
            if (rstd) rstd[row] = r;
        }
    }
}

template <class Ty>
__global__ __launch_bounds__(kLongThreads) void k_layernorm_long_dx(NormArgs a, const typename Ty::T *g,
                                                                    const float *mean, const float *rstd,
                                                                    typename Ty::T *dx) {
    __shared__ float sh[2 * kLongThreads / 64];
    TeamSum<kLongThreads> sum{sh};
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const typename Ty::T *x = (const typename Ty::T *)a.x + row * a.D, *gr = g + row * a.D;
        const size_t wr = (row % a.G) * a.D;
        const float m = mean[row], r = rstd[row];
        float s1 = 0.f, s2 = 0.f;
        for (int i = threadIdx.x; i < a.D; i += kLongThreads) {
            const float u = Ty::up(gr[i]) * weight_at(a, a.w, wr + i, 1.f), xh = (Ty::up(x[i]) - m) * r;
            s1 += u;
            s2 = fmaf(u, xh, s2);
        }
        s1 = sum(s1) / (float)a.D;
        s2 = sum(s2) / (float)a.D;
        for (int i = threadIdx.x; i < a.D; i += kLongThreads) {
            const float u = Ty::up(gr[i]) * weight_at(a, a.w, wr + i, 1.f), xh = (Ty::up(x[i]) - m) * r;
            dx[row * a.D + i] = Ty::down(r * (u - s1 - xh * s2));
        }
    }
}

// one column per thread; partial blockIdx.y G + group of the group's rows blockIdx.y, blockIdx.y + kLongSplits, ...
template <class Ty>
__global__ __launch_bounds__(256) void k_layernorm_long_part(NormArgs a, const typename Ty::T *g, const float *mean,
                                                             const float *rstd, float *part) {
    const int n = a.G * a.D, i = blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int grp = i / a.D, c = i % a.D;
    float sw = 0.f, sb = 0.f;
    for (size_t row = grp + (size_t)a.G * blockIdx.y; row < a.rows; row += (size_t)a.G * kLongSplits) {
        const float gv = Ty::up(g[row * a.D + c]);
        sw = fmaf(gv, (Ty::up(((const typename Ty::T *)a.x)[row * a.D + c]) - mean[row]) * rstd[row], sw);
        sb += gv;
    }
    float *p = part + ((size_t)blockIdx.y * a.G + grp) * 2 * a.D + c;
    p[0] = sw;
    p[a.D] = sb;
}

// ---- launches -------------------------------------------------------------------------------------

// threads per row and units per thread: two units where a row has them, so that enough is in flight
// (rows of 2048 in bf16: 53 us with 128 threads, 62 us with 256 of one unit).  1024 threads have 128
// registers each, which hold 16 elements a thread, but for the adjoint, with six float32 values for
// each, not the next row as well: it takes 512 threads where these can hold the row (4096 rows of
// 16384 in bf16: 105 us for 144; forwards 65 for 59).  0: none holds the row
struct NormShape {
    int team, nv;
};
static NormShape shape_of(int dtype, int D, bool adjoint) {
    const int e = dtype == DEER_F32 ? 4 : 8, u = (D + e - 1) / e;
    if (u <= 16) return {16, 1};
    if (u <= 64) return {64, 1};
    if (u <= 128) return {64, 2};
    if (u <= 256) return {128, 2};
    if (u <= 512) return {256, 2};
    if (u <= 1024) return {512, 2};
    if (u <= 2048) return adjoint ? NormShape{512, 4} : NormShape{1024, 2};
    if (u <= 4096 && dtype == DEER_F32) return {1024, 4};
    return {0, 0};
}

// teams: as many as fill the chip with `threads` threads, whole groups of rows
static int teams_of(size_t rows, int G, int team, size_t threads) {
    const size_t cap = threads / team;
    if (rows <= cap) return (int)rows;
    return (int)(cap < (size_t)G ? (size_t)G : cap / G * G);
}
// (with 3/4, 1, 3/2 and 2 times as many, 32768 rows in bf16 take, of 2048 forwards, 55, 53, 57 and 64 us, of
// 4096 backwards 171, 162, 170 and 188)
constexpr size_t kForwardThreads = 256 * 1024, kAdjointThreads = 256 * 512;

static int partials_of(const NormArgs &a) {
    const NormShape s = shape_of(a.dtype, a.D, true);
    if (!s.team) return kLongSplits * a.G;
    const int nt = teams_of(a.rows, a.G, s.team, kAdjointThreads), tpb = block_of(s.team) / s.team;
    return a.G > 1 ? nt : (nt + tpb - 1) / tpb;
}

template <int N>
using Int = std::integral_constant<int, N>;

template <bool ADJOINT, class Fn>
static int with_shape(const NormArgs &a, Fn f) {
    const NormShape s = shape_of(a.dtype, a.D, ADJOINT);
    return with_dtype(a.dtype, [&](auto ty) {
        if (s.team == 16) return f(ty, Int<16>{}, Int<1>{});
        if (s.team == 64) return s.nv == 1 ? f(ty, Int<64>{}, Int<1>{}) : f(ty, Int<64>{}, Int<2>{});
        if (s.team == 128) return f(ty, Int<128>{}, Int<2>{});
        if (s.team == 256) return f(ty, Int<256>{}, Int<2>{});
        if (s.team == 512 && s.nv == 2) return f(ty, Int<512>{}, Int<2>{});
        if constexpr (std::is_same<decltype(ty), F32>::value)
            if (s.nv == 4 && s.team == 1024) return f(ty, Int<1024>{}, Int<4>{});
        if constexpr (ADJOINT) return f(ty, Int<512>{}, Int<4>{});
        else return f(ty, Int<1024>{}, Int<2>{});
    });
}

// whether every row of x, p and q starts on a unit's boundary
static bool units_whole(const NormArgs &a, const void *p, const void *q) {
    return ((uintptr_t)a.x % 16 | (uintptr_t)p % 16 | (uintptr_t)q % 16) == 0 &&
           a.D % (16 / (int)dtype_size(a.dtype)) == 0;
}

int launch_layernorm(const NormArgs &a, void *y, float *mean, float *rstd, hipStream_t st) {
    const NormShape s = shape_of(a.dtype, a.D, false);
    KTimer kt("k_layernorm", st);
    if (!s.team)
        return with_dtype(a.dtype, [&](auto ty) {
            using Ty = decltype(ty);
            hipLaunchKernelGGL(k_layernorm_long<Ty>, dim3((unsigned)(a.rows < 4096 ? a.rows : 4096)), dim3(kLongThreads),
                               0, st, a, (typename Ty::T *)y, mean, rstd);
            DEER_LAUNCH_CHECK("k_layernorm_long");
            return (int)DEER_OK;
        });
    const int nt = teams_of(a.rows, a.G, s.team, kForwardThreads);
    return with_shape<false>(a, [&](auto ty, auto team, auto nv) {
        using Ty = decltype(ty);
        constexpr int TEAM = decltype(team)::value, NV = decltype(nv)::value, TPB = block_of(TEAM) / TEAM;
        hipLaunchKernelGGL((k_layernorm<Ty, TEAM, NV>), dim3((nt + TPB - 1) / TPB), dim3(block_of(TEAM)), 0, st, a, nt,
                           units_whole(a, y, nullptr), (typename Ty::T *)y, mean, rstd);
        DEER_LAUNCH_CHECK("k_layernorm");
        return (int)DEER_OK;
    });
}

size_t layernorm_adjoint_ws_bytes(const NormArgs &a) { return (size_t)partials_of(a) * 2 * a.D * sizeof(float); }

static int launch_sum(const NormArgs &a, const float *part, float *dw, float *db, hipStream_t st) {
    KTimer kt("k_layernorm_sum", st);
    const int np = partials_of(a);
    const dim3 grid((unsigned)(a.G * ((a.D + 31) / 32)), 2);
    if (np / a.G > 128) hipLaunchKernelGGL(k_layernorm_sum<32>, grid, dim3(1024), 0, st, a.G, a.D, np, part, dw, db);
    else hipLaunchKernelGGL(k_layernorm_sum<8>, grid, dim3(256), 0, st, a.G, a.D, np, part, dw, db);
    DEER_LAUNCH_CHECK("k_layernorm_sum");
    return DEER_OK;
}

int launch_layernorm_adjoint(const NormArgs &a, const void *g, const float *mean, const float *rstd, void *dx,
                             float *dw, float *db, void *ws, hipStream_t st) {
    const NormShape s = shape_of(a.dtype, a.D, true);
    const bool sums = dw || db;
    float *part = sums ? (float *)ws : nullptr;
    int rc;
    if (!s.team) {
        rc = with_dtype(a.dtype, [&](auto ty) {
            using Ty = decltype(ty);
            using T = typename Ty::T;
            if (dx) {
                KTimer kt("k_layernorm_dx", st);
                hipLaunchKernelGGL(k_layernorm_long_dx<Ty>, dim3((unsigned)(a.rows < 4096 ? a.rows : 4096)),
                                   dim3(kLongThreads), 0, st, a, (const T *)g, mean, rstd, (T *)dx);
                DEER_LAUNCH_CHECK("k_layernorm_long_dx");
            }
            if (!sums) return (int)DEER_OK;
            KTimer kt("k_layernorm_part", st);
            hipLaunchKernelGGL(k_layernorm_long_part<Ty>, dim3((unsigned)((a.G * a.D + 255) / 256), kLongSplits), dim3(256),
                               0, st, a, (const T *)g, mean, rstd, part);
            DEER_LAUNCH_CHECK("k_layernorm_long_part");
            return (int)DEER_OK;
        });
    } else {
        const int nt = teams_of(a.rows, a.G, s.team, kAdjointThreads);
        rc = with_shape<true>(a, [&](auto ty, auto team, auto nv) {
            using Ty = decltype(ty);
            using T = typename Ty::T;
            constexpr int TEAM = decltype(team)::value, NV = decltype(nv)::value, TPB = block_of(TEAM) / TEAM;
            KTimer kt("k_layernorm_adj", st);
            hipLaunchKernelGGL((k_layernorm_adj<Ty, TEAM, NV>), dim3((nt + TPB - 1) / TPB), dim3(block_of(TEAM)), 0, st, a,
                               nt, units_whole(a, g, dx), (const T *)g, mean, rstd, (T *)dx, part);
            DEER_LAUNCH_CHECK("k_layernorm_adj");
            return (int)DEER_OK;
        });
    }
    if (rc || !sums) return rc;
    return launch_sum(a, part, dw, db, st);
}

}  // namespace deer
