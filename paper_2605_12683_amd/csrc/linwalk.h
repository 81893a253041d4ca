// The walk of linear attention on the matrix cores (internal to libdeer, not part of the ABI):
//   S_t = a_t S_{t-1} + k_t v_t^T,  o_t = S_t^T q_t
// for every step of a sequence, C steps at a time.  With c_i the log decay summed from the chunk's
// first step to step i (in it), L over the whole chunk and S the state entering it,
//   o_i  = exp(c_i) S^T q_i + sum_{j <= i} exp(c_i - c_j) (k_j q_i) v_j
//   S   <- exp(L) S + sum_j k_j (exp(L - c_j) v_j)^T.
// Every exponent is a difference that no decay makes positive, so nothing overflows however small
// the decays are (factoring exp(c_i) exp(-c_j) would); the sums c are taken in float64 and kept as
// two floats, so that a difference of two large sums of near size is exact to float32.
//
// Products run on the bf16 matrix cores with float32 sums.  Operands of fewer bits enter exactly: a
// bf16 number as it is, an fp16 number as two bf16 parts, a float32 number as three (split16.h).
// What is formed in between is split likewise, into NPX parts where it meets the outputs (two: 16
// bits, for 16-bit outputs, 2^8 times finer than their own rounding; three: float32's 24) and always
// into three where it enters the state, which is float32 for as long as the sequence lasts.
//
// One block of four waves walks one head's chunks for NB = 4 CW columns of the state; a wave keeps
// its CW columns in registers for the whole walk, as matrix-core accumulators.  Their lane layout
// (rows 4 g + r, column c of lane 16 g + c) is also that of an operand with the rows as the summed
// index, if the other operand lists them in the order 4 g + 0..3, 16 + 4 g + 0..3 of each 32: q is
// stored in LDS in that order, and the state enters its product with no exchange between lanes.  k
// and v lie in LDS as they are and are read row-wise or, where steps are the summed index,
// transposed by ds_read_b64_tr_b16.  The decayed scores, formed by the four waves tile by tile (those
// on and below the diagonal), are exchanged through LDS in operand order.
//
// What bounds it: a chunk of 64 steps at Kd = N = 128 in bf16 moves 64 KiB and takes 194 matrix
// instructions of 16 x 16 x 32 a wave (1.5 us at their rate, against 3.3 us for the bytes at 5 TB/s
// with all 256 CUs walking), so memory, as long as latencies are hidden: the next chunk's rows are
// loaded into registers while this one is computed (barriers order LDS only), and tiles are kept
// below 80 KiB of LDS, C = 32 instead of 64 where needed, so that two blocks share a CU.
#pragma once

#include "launch.h"
#include "split16.h"
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

// log decay whose factor the walk applies to its state on entering step t: forwards that of t,
// backwards that of t + 1; 0 (a factor of one) behind the sequence's end
__device__ __forceinline__ float gate_raw(const LinArgs &a, int b, int h, int t, int len, bool rev) {
    const int s = rev ? t + 1 : t;
    if (s >= len || s < 0) return 0.f;
    return a.per_step ? a.log_decay[((size_t)b * a.T + s) * a.H + h] : a.log_decay[h];
}

__device__ __forceinline__ int length_of(const LinArgs &a, int b) {
    if (!a.lengths) return a.T;
    const int n = a.lengths[b];
    return n < 0 ? 0 : (n > a.T ? a.T : n);
}

// ---- tile shapes -------------------------------------------------------------------------------

template <class Ty>
struct InParts;   // bf16 parts that hold an operand exactly
template <>
struct InParts<Bf16> { static constexpr int n = 1; };
template <>
struct InParts<F16> { static constexpr int n = 2; };
template <>
struct InParts<F32> { static constexpr int n = 3; };

// padded width of the summed side, and columns per wave: 32 where the state then fits the registers
// (Kd <= 128) and the columns fill more than half a block; 16 with float32 tiles of 128, whose LDS
// tiles would leave one block to a CU
constexpr int kt_of(int Kd) { return Kd <= 32 ? 32 : Kd <= 64 ? 64 : Kd <= 128 ? 128 : 256; }
constexpr int cw_of(int parts, int KT, int N) { return N > 64 && KT <= (parts == 3 ? 64 : 128) ? 32 : 16; }

template <int NPI, int KT, int CW, int NPX, bool OUT>
struct LinTile {
    static constexpr int NB = 4 * CW;
    static constexpr int PQ = KT + 8, PK = KT + 16, PV = NB + 16;   // LDS row pitches: no bank conflicts
    static constexpr int bytes(int C) {
        return NPI * C * 2 * ((OUT ? PQ : 0) + PK + PV) + (OUT ? (C / 16) * (C / 32) * NPX * 1024 : 0) +
               2 * (4 * C + 4) * 4 + 4 * C * 4;
    }
    static constexpr int C = bytes(64) <= 80 * 1024 ? 64 : 32;
    static constexpr int lds = bytes(C);
    static constexpr int waves = lds <= 80 * 1024 ? 2 : 1;          // per SIMD
};

struct LinRoles {
    LinRole r[3];
};

// ---- loads of a chunk's rows -----------------------------------------------------------------

typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef short v4s __attribute__((ext_vector_type(4)));

// W columns of C rows, NU units of 16 bytes a thread
template <class Ty, int C, int W>
struct RowTile {
    static constexpr int E = 16 / sizeof(typename Ty::T), UPR = W / E, NU = (C * UPR + 255) / 256;
    v4u u[NU];

    __device__ __forceinline__ void load(const typename Ty::T *base, long st, int t0, bool rev, int len, int col0,
                                         int width, bool vec) {
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int n = i * 256 + threadIdx.x, row = n / UPR, d = (n % UPR) * E;
            const int t = rev ? t0 + C - 1 - row : t0 + row;
            u[i] = v4u{0, 0, 0, 0};
            if ((C * UPR % 256 == 0 || row < C) && t < len) u[i] = load_unit<Ty>(base + t * st, col0 + d, width, vec);
        }
    }

    // planes of bf16 parts [C][pitch]; PERM: the columns of each 32 in the order 4 g + 0..3, 16 + 4 g + 0..3
    template <bool PERM>
    __device__ __forceinline__ void store(uint16_t *lds, int pitch) const {
        constexpr int NP = InParts<Ty>::n;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int n = i * 256 + threadIdx.x, row = n / UPR, d = (n % UPR) * E;
            if (C * UPR % 256 != 0 && row >= C) continue;
#pragma unroll
            for (int half = 0; half < E / 4; ++half) {   // four elements at a time
                uint32_t p[NP][2];
                parts(u[i], half, p);
                const int e = d + 4 * half;
                const int at = PERM ? (e & ~31) + ((e & 15) >> 2) * 8 + ((e >> 4) & 1) * 4 : e;
#pragma unroll
                for (int q = 0; q < NP; ++q)
                    *(v2u *)(lds + (q * C + row) * pitch + at) = v2u{p[q][0], p[q][1]};
            }
        }
    }

    template <int NP>
    static __device__ __forceinline__ void parts(v4u u, int half, uint32_t (&p)[NP][2]) {
        if constexpr (NP == 1) {
            p[0][0] = u[2 * half], p[0][1] = u[2 * half + 1];
        } else {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                float x0, x1;
                if constexpr (NP == 2) {
                    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
                    const v2h h = __builtin_bit_cast(v2h, (uint32_t)u[2 * half + w]);
                    x0 = (float)h[0], x1 = (float)h[1];
                } else {
                    x0 = __uint_as_float(u[2 * w]), x1 = __uint_as_float(u[2 * w + 1]);
                }
                uint32_t s[3];
                split_pair(x0, x1, s);
#pragma unroll
                for (int q = 0; q < NP; ++q) p[q][w] = s[q];
            }
        }
    }
};

// four rows of one column: lane 16 g + c of a wave gets rows row0 + 4 g + 0..3 of column col0 + c
__device__ __forceinline__ v2u read_turned(const uint16_t *lds, int pitch, int row0, int col0, int g, int c) {
    const uint16_t *p = lds + (row0 + 4 * g + (c >> 2)) * pitch + col0 + 4 * (c & 3);
    return __builtin_bit_cast(
        v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)p));
}

// the first NP parts of eight floats, as one operand each
template <int NP>
__device__ __forceinline__ void split8(const float (&x)[8], v4u (&p)[NP]) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        float x0 = x[2 * w], x1 = x[2 * w + 1];
#pragma unroll
        for (int q = 0; q < NP; ++q) {
            const uint32_t s = cvt_pair(x0, x1);
            p[q][w] = s;
            if (q + 1 < NP) {
                x0 -= __uint_as_float(s << 16);
                x1 -= __uint_as_float(s & 0xffff0000u);
            }
        }
    }
}

// acc += sum of the products of parts whose indices add up to at most LIM, the smallest first
template <int LIM, int NA, int NB>
__device__ __forceinline__ v4f mfma_parts(const v4u (&x)[NA], const v4u (&y)[NB], v4f acc) {
#pragma unroll
    for (int s = LIM; s >= 0; --s)
#pragma unroll
        for (int p = 0; p < NA; ++p) {
            const int q = s - p;
            if (q >= 0 && q < NB) acc = mfma_b(x[p], y[q], acc);
        }
    return acc;
}

// ---- decays of a chunk --------------------------------------------------------------------------

template <int C>
struct Decays {
    float hi[C], lo[C];   // log2 decay summed up to each step
    float into[C];        // sc_kv exp2(L - c): what a step's k v^T has left at the chunk's end
    float from[C];        // exp2(c): what the entering state has left at each step
    float all;            // exp2(L)
    float pad[3];
};

// by one wave; raw: this lane's log decay (lanes beyond C repeat the others).  Returns L.
template <int C>
__device__ __forceinline__ double chunk_decays(Decays<C> &d, float raw, float sc_kv) {
    const int lane = threadIdx.x & 63, i = lane & (C - 1);
    double s = gate_of(raw);
#pragma unroll
    for (int off = 1; off < C; off <<= 1) {
        const double o = __shfl_up(s, off, C);
        if (i >= off) s += o;
    }
    const double L = __shfl(s, C - 1, C);
    const float hi = (float)s;
    d.hi[i] = hi;
    d.lo[i] = (float)(s - (double)hi);
    d.into[i] = sc_kv * __builtin_amdgcn_exp2f((float)(L - s));
    d.from[i] = __builtin_amdgcn_exp2f(hi);
    if (i == 0) d.all = __builtin_amdgcn_exp2f((float)L);
    return L;
}

// ---- the walk ---------------------------------------------------------------------------------

// OUT: outputs (and the last state, dots, anchors) of each segment from the state entering it;
// otherwise the state that each segment adds by itself, from zero, and its decay.
template <class Ty, int KT, int CW, int NPX, bool OUT>
__global__ __launch_bounds__(256, (LinTile<InParts<Ty>::n, KT, CW, NPX, OUT>::waves)) void k_lin_walk(LinArgs a,
                                                                                                     LinRoles rs) {
    constexpr int NPI = InParts<Ty>::n;
    using Tile = LinTile<NPI, KT, CW, NPX, OUT>;
    using T = typename Ty::T;
    constexpr int C = Tile::C, NB = Tile::NB, PQ = Tile::PQ, PK = Tile::PK, PV = Tile::PV;
    constexpr int NT = C / 16, KS = C / 32, DT = KT / 16, CT = CW / 16;
    extern __shared__ __align__(16) unsigned char smem[];
    uint16_t *Ks = (uint16_t *)smem, *Vs = Ks + NPI * C * PK, *Qs = Vs + NPI * C * PV;
    unsigned char *rest = (unsigned char *)(Qs + (OUT ? NPI * C * PQ : 0));
    v4u *Ps = (v4u *)rest;                                     // [NT][KS][NPX][64 lanes]
    Decays<C> *dec = (Decays<C> *)(rest + (OUT ? NT * KS * NPX * 1024 : 0));
    float *dots = (float *)(dec + 2);                          // [4][C]

    const LinRole &ro = rs.r[blockIdx.y];
    const int tiles = (ro.N + NB - 1) / NB;
    const long units = (long)a.B * a.H * a.nseg * tiles;
    if ((long)blockIdx.x >= units) return;
    const int tile = blockIdx.x % tiles, seg = blockIdx.x / tiles % a.nseg, bh = blockIdx.x / tiles / a.nseg;
    const int b = bh / a.H, h = bh % a.H;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const bool rev = ro.reverse;
    const int len = length_of(a, b);
    const int lo = seg * a.seg_steps, hi = lo + a.seg_steps < a.T ? lo + a.seg_steps : a.T;
    const int chunks = (hi - lo + C - 1) / C;
    const size_t mat = (size_t)ro.Kd * ro.N;
    const int col0 = tile * NB, n0 = col0 + w * CW;            // the block's and the wave's first column

    // the segment that comes last adds to no other: its own sum is needed for the last state only
    if (!OUT && seg == (rev ? 0 : a.nseg - 1) && !ro.fin) return;

    const T *qb = (const T *)ro.q.p + b * ro.q.sb + (h / ro.q.r) * ro.q.sh;
    const T *kb = (const T *)ro.k.p + b * ro.k.sb + (h / ro.k.r) * ro.k.sh;
    const T *vb = (const T *)ro.v.p + b * ro.v.sb + (h / ro.v.r) * ro.v.sh;
    constexpr int E = 16 / sizeof(T);
    auto wide = [](const T *p, long st, int n) { return (((uintptr_t)p | (uintptr_t)(st * sizeof(T))) & 15) == 0 && n % E == 0; };
    const bool qw = OUT && wide(qb, ro.q.st, ro.Kd), kw = wide(kb, ro.k.st, ro.Kd), vw = wide(vb, ro.v.st, ro.N);

    RowTile<Ty, C, KT> qr, kr;
    RowTile<Ty, C, NB> vr;
    auto t0_of = [&](int n) { return lo + (rev ? chunks - 1 - n : n) * C; };
    auto load = [&](int n) {
        const int t0 = t0_of(n);
        kr.load(kb, ro.k.st, t0, rev, len, 0, ro.Kd, kw);
        vr.load(vb, ro.v.st, t0, rev, len, col0, ro.N, vw);
        if constexpr (OUT) qr.load(qb, ro.q.st, t0, rev, len, 0, ro.Kd, qw);
    };
    auto gate = [&](int n) {
        if (n >= chunks) return 0.f;
        const int i = lane & (C - 1);
        return gate_raw(a, b, h, t0_of(n) + (rev ? C - 1 - i : i), len, rev);
    };

    v4f S[DT][CT];
    {
        const float *src = nullptr;
        int sd = 0, sn = 0;
        if (OUT) {
            if (a.nseg > 1) src = ro.seg + ((size_t)bh * a.nseg + seg) * mat, sd = ro.seg_d, sn = ro.seg_n;
            else if (ro.init) src = ro.init + bh * mat, sd = ro.init_d, sn = ro.init_n;
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int d = dt * 16 + 4 * g + r, n = n0 + ct * 16 + c;
                    S[dt][ct][r] = src && d < ro.Kd && n < ro.N ? src[(size_t)d * sd + (size_t)n * sn] : 0.f;
                }
    }
    auto put_state = [&](float *dst, int sd, int sn, float f) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int d = dt * 16 + 4 * g + r, n = n0 + ct * 16 + c;
                    if (d < ro.Kd && n < ro.N) dst[(size_t)d * sd + (size_t)n * sn] = f * S[dt][ct][r];
                }
    };

    // tiles above the diagonal that share an operand with one on it stay zero
    if constexpr (OUT)
        for (int i = threadIdx.x; i < NT * KS * NPX * 64; i += 256) Ps[i] = v4u{0, 0, 0, 0};
    load(0);
    double total = 0.0;                                        // wave 3: log2 decay of the segment
    float raw = 0.f;
    if (w == 3) {
        total += chunk_decays<C>(dec[0], gate(0), ro.sc_kv);
        raw = gate(1);
    }
    const int na = (a.T + kLinAnchor - 1) / kLinAnchor;

    for (int n = 0; n < chunks; ++n) {
        const int t0 = t0_of(n);
        const Decays<C> &dc = dec[n & 1];
        kr.template store<false>(Ks, PK);
        vr.template store<false>(Vs, PV);
        if constexpr (OUT) qr.template store<true>(Qs, PQ);
        lds_barrier();
        if (n + 1 < chunks) {
            load(n + 1);
            if (w == 3) {
                total += chunk_decays<C>(dec[(n + 1) & 1], raw, ro.sc_kv);
                raw = gate(n + 2);
            }
        }
        float *anc = nullptr;
        if (OUT && ro.anchor && ((t0 + C) % kLinAnchor == 0 || t0 + C >= a.T))
            anc = ro.anchor + ((size_t)bh * na + t0 / kLinAnchor) * mat;
        if (OUT && anc && rev) put_state(anc, ro.N, 1, 1.f);

        v4f O[NT][CT];
        if constexpr (OUT) {
            // decayed scores, transposed: rows j, columns i
            for (int tl = w; tl < NT * (NT + 1) / 2; tl += 4) {
                const int it = tl >= 6 ? 3 : tl >= 3 ? 2 : tl >= 1 ? 1 : 0, jt = tl - it * (it + 1) / 2;
                v4f acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int u = 0; u < KT / 32; ++u) {
                    v4u kf[NPI], qf[NPI];
#pragma unroll
                    for (int p = 0; p < NPI; ++p) {
                        const uint16_t *kp = Ks + (p * C + jt * 16 + c) * PK + u * 32 + 4 * g;
                        const v2u k0 = *(const v2u *)kp, k1 = *(const v2u *)(kp + 16);
                        kf[p] = v4u{k0[0], k0[1], k1[0], k1[1]};
                        qf[p] = *(const v4u *)(Qs + (p * C + it * 16 + c) * PQ + u * 32 + 8 * g);
                    }
                    acc = mfma_parts<NPI - 1>(kf, qf, acc);
                }
                const int i = it * 16 + c, j0 = jt * 16 + 4 * g;
                const float hi_i = dc.hi[i], lo_i = dc.lo[i];
                float x[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float e = (hi_i - dc.hi[j0 + r]) + (lo_i - dc.lo[j0 + r]);
                    const float p = acc[r] * ro.sc_kv * __builtin_amdgcn_exp2f(e);
                    x[r] = j0 + r <= i ? p : 0.f;
                }
                uint32_t *dst = (uint32_t *)(Ps + ((it * KS + (jt >> 1)) * NPX) * 64 + lane) + (jt & 1) * 2;
                uint32_t p0[3], p1[3];
                split_pair(x[0], x[1], p0);
                split_pair(x[2], x[3], p1);
#pragma unroll
                for (int q = 0; q < NPX; ++q) *(v2u *)(dst + q * 64 * 4) = v2u{p0[q], p1[q]};
            }
            // what the entering state gives, transposed: rows n, columns i
#pragma unroll
            for (int it = 0; it < NT; ++it)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) O[it][ct] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < KT / 32; ++u) {
                v4u sf[CT][NPX];
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    float x[8];
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] = S[2 * u][ct][r], x[4 + r] = S[2 * u + 1][ct][r];
                    split8<NPX>(x, sf[ct]);
                }
#pragma unroll
                for (int it = 0; it < NT; ++it) {
                    v4u qf[NPI];
#pragma unroll
                    for (int p = 0; p < NPI; ++p) qf[p] = *(const v4u *)(Qs + (p * C + it * 16 + c) * PQ + u * 32 + 8 * g);
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) O[it][ct] = mfma_parts<NPX - 1>(sf[ct], qf, O[it][ct]);
                }
            }
#pragma unroll
            for (int it = 0; it < NT; ++it) {
                const float f = dc.from[it * 16 + c];
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) O[it][ct] *= f;
            }
            lds_barrier();
        }

        // the chunk's own steps, and the state at its end
        const float all = dc.all;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) S[dt][ct] *= all;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            v4u vf[CT][NPI], sv[CT][3];
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = 0.f;
#pragma unroll
                for (int p = 0; p < NPI; ++p) {
                    const uint16_t *vp = Vs + p * C * PV;
                    const v2u v0 = read_turned(vp, PV, ks * 32, w * CW + ct * 16, g, c);
                    const v2u v1 = read_turned(vp, PV, ks * 32 + 16, w * CW + ct * 16, g, c);
                    vf[ct][p] = v4u{v0[0], v0[1], v1[0], v1[1]};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[2 * e] += __uint_as_float(vf[ct][p][e] << 16);
                        x[2 * e + 1] += __uint_as_float(vf[ct][p][e] & 0xffff0000u);
                    }
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x[r] *= dc.into[ks * 32 + 4 * g + r];
                    x[4 + r] *= dc.into[ks * 32 + 16 + 4 * g + r];
                }
                split8<3>(x, sv[ct]);
            }
            if constexpr (OUT) {
#pragma unroll
                for (int it = 2 * ks; it < NT; ++it) {
                    v4u pf[NPX];
#pragma unroll
                    for (int q = 0; q < NPX; ++q) pf[q] = Ps[((it * KS + ks) * NPX + q) * 64 + lane];
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) O[it][ct] = mfma_parts<NPX - 1>(vf[ct], pf, O[it][ct]);
                }
            }
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                v4u kf[NPI];
#pragma unroll
                for (int p = 0; p < NPI; ++p) {
                    const uint16_t *kp = Ks + p * C * PK;
                    const v2u k0 = read_turned(kp, PK, ks * 32, dt * 16, g, c);
                    const v2u k1 = read_turned(kp, PK, ks * 32 + 16, dt * 16, g, c);
                    kf[p] = v4u{k0[0], k0[1], k1[0], k1[1]};
                }
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) S[dt][ct] = mfma_parts<2>(kf, sv[ct], S[dt][ct]);
            }
        }

        if constexpr (OUT) {
#pragma unroll
            for (int it = 0; it < NT; ++it) {
                const int i = it * 16 + c, t = rev ? t0 + C - 1 - i : t0 + i;
                const bool live = t < len;
                float dot = 0.f;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    const int nn = n0 + ct * 16 + 4 * g;
                    v4f o = O[it][ct] * ro.sc_o;
                    if (!live) o = v4f{0.f, 0.f, 0.f, 0.f};
                    if (t < a.T && nn < ro.N) {
                        const size_t at = (((size_t)b * a.T + t) * a.H + h) * ro.N + nn;
                        if (ro.out_f32) {
                            float *p = (float *)ro.out + at;
                            if (ro.N % 4 == 0) *(v4f *)p = o;
                            else
                                for (int r = 0; r < 4; ++r)
                                    if (nn + r < ro.N) p[r] = o[r];
                        } else {
                            T *p = (T *)ro.out + at;
                            typedef T v4t __attribute__((ext_vector_type(4)));
                            const v4t y = {Ty::down(o[0]), Ty::down(o[1]), Ty::down(o[2]), Ty::down(o[3])};
                            if (ro.wide_out) *(v4t *)p = y;
                            else
                                for (int r = 0; r < 4; ++r)
                                    if (nn + r < ro.N) p[r] = y[r];
                        }
                    }
                    if (ro.dot && live) {
                        const T *p = (const T *)ro.partner.p + b * ro.partner.sb + t * ro.partner.st +
                                     (h / ro.partner.r) * ro.partner.sh + nn;
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (nn + r < ro.N) dot = fmaf(o[r], Ty::up(p[r]), dot);
                    }
                }
                if (ro.dot) {
                    dot = group_sum(dot);
                    if (g == 0) dots[w * C + i] = dot;
                }
            }
        }
        if (OUT && anc && !rev) put_state(anc, ro.N, 1, 1.f);
        lds_barrier();
        if (OUT && ro.dot && (int)threadIdx.x < C) {
            const int i = threadIdx.x, t = rev ? t0 + C - 1 - i : t0 + i;
            if (t < a.T)
                ro.dot[((size_t)tile * a.B * a.H + bh) * a.T + t] =
                    (dots[i] + dots[C + i]) + (dots[2 * C + i] + dots[3 * C + i]);
        }
    }

    if constexpr (OUT) {
        if (ro.fin && a.nseg == 1) {
            const float f = rev ? __builtin_amdgcn_exp2f((float)gate_of(gate_raw(a, b, h, -1, len, true))) : 1.f;
            put_state(ro.fin + bh * mat, ro.fin_d, ro.fin_n, f);
        }
    } else {
        put_state(ro.seg + ((size_t)bh * a.nseg + seg) * mat, ro.N, 1, 1.f);
        if (w == 3 && lane == 0 && tile == 0) ro.seg_decay[(size_t)bh * a.nseg + seg] = __builtin_amdgcn_exp2f((float)total);
    }
}

// ---- launches -------------------------------------------------------------------------------------

template <class Ty, int KT, int CW, int NPX, bool OUT>
int launch_walk_tile(const LinArgs &a, const LinRole *roles, int n, hipStream_t st) {
    using Tile = LinTile<InParts<Ty>::n, KT, CW, NPX, OUT>;
    LinRoles rs{};
    int tiles = 0;
    for (int i = 0; i < n; ++i) {
        rs.r[i] = roles[i];
        const int t = (roles[i].N + Tile::NB - 1) / Tile::NB;
        tiles = t > tiles ? t : tiles;
    }
    const void *fn = (const void *)k_lin_walk<Ty, KT, CW, NPX, OUT>;
    if (Tile::lds > 64 * 1024) DEER_HIP(hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, Tile::lds));
    KTimer kt(OUT ? "k_lin_walk" : "k_lin_walk_states", st);
    hipLaunchKernelGGL((k_lin_walk<Ty, KT, CW, NPX, OUT>), dim3((unsigned)(a.B * a.H * a.nseg * tiles), n), dim3(256),
                       Tile::lds, st, a, rs);
    DEER_LAUNCH_CHECK("k_lin_walk");
    return DEER_OK;
}

template <class Ty, int NPX, bool OUT>
int launch_walk_parts(const LinArgs &a, const LinRole *roles, int n, hipStream_t st) {
    constexpr int NPI = InParts<Ty>::n;
    const int KT = kt_of(roles[0].Kd), CW = cw_of(NPI, KT, roles[0].N);
    if (KT == 256) return launch_walk_tile<Ty, 256, 16, NPX, OUT>(a, roles, n, st);
    if (CW == 16) {
        if (KT == 32) return launch_walk_tile<Ty, 32, 16, NPX, OUT>(a, roles, n, st);
        if (KT == 64) return launch_walk_tile<Ty, 64, 16, NPX, OUT>(a, roles, n, st);
        return launch_walk_tile<Ty, 128, 16, NPX, OUT>(a, roles, n, st);
    }
    if (KT == 32) return launch_walk_tile<Ty, 32, 32, NPX, OUT>(a, roles, n, st);
    if (KT == 64) return launch_walk_tile<Ty, 64, 32, NPX, OUT>(a, roles, n, st);
    if constexpr (NPI < 3) return launch_walk_tile<Ty, 128, 32, NPX, OUT>(a, roles, n, st);
    return DEER_ERR_INVALID_ARG;
}

}  // namespace deer
