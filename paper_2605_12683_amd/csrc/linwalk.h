// The walk of linear attention on the matrix cores (internal to libdeer, not part of the ABI):
//   S_t = a_t S_{t-1} + k_t v_t^T,  o_t = S_t^T q_t
// for every step of a sequence, C steps at a time.  With c_i the log decay summed from the chunk's
// first step to step i (in it), L over the whole chunk and S the state entering it,
//   o_i  = exp(c_i) S^T q_i + sum_{j <= i} exp(c_i - c_j) (k_j q_i) v_j
//   S   <- exp(L) S + sum_j k_j (exp(L - c_j) v_j)^T.
// Every exponent is a difference that no decay makes positive (but for the half that Decays speaks of),
// so nothing overflows however small the decays are (factoring exp(c_i) exp(-c_j) would); the sums c
// are taken in float64 and kept as two floats, so that a difference of two large sums of near size is
// exact to float32.
//
// Products run on the bf16 matrix cores with float32 sums.  Operands of fewer bits enter exactly: a
// bf16 number as it is, an fp16 number as two bf16 parts, a float32 number as three (split16.h).
// What is formed in between (the decayed scores, the entering state, v times its decay) is float32 and
// enters the next product in three parts, which hold all its 24 bits whatever the operands' type. (Two
// parts where it meets 16-bit outputs would save up to 8% of the time in bf16 and 12% in fp16, but flip
// the last bit of 0.24% of the outputs in bf16, and of over 1% in fp16, against sums in float32.)
//
// One block of NW waves walks one head's chunks for NB = 16 NW CT columns of the state; a wave keeps
// its 16 CT columns in registers for the whole walk, as matrix-core accumulators.  Their lane layout
// (rows 4 g + r, column c of lane 16 g + c) is also that of an operand with the rows as the summed
// index, if the other operand lists them in the order 4 g + 0..3, 16 + 4 g + 0..3 of each 32: q is
// stored in LDS in that order, and the state enters its product with no exchange between lanes.  k
// and v lie in LDS as they are and are read row-wise or, where steps are the summed index,
// transposed by ds_read_b64_tr_b16.  The decayed scores, formed by the four waves tile by tile (those
// on and below the diagonal), are exchanged through LDS in operand order.
//
// What bounds it: a chunk of 64 steps at Kd = N = 128 in bf16 moves 64 KiB and takes 238 matrix
// instructions of 16 x 16 x 32 a wave (1.9 us at their rate, against 3.3 us for the bytes at 5 TB/s
// with all 256 CUs walking).  Between them stand the vector instructions that split and scale what is
// formed in between: of the issue cycles, vector and matrix instructions fill 62 + 29% (32 heads of
// 64 x 64, 65536 steps, 768 blocks: 250 us, 2.7 TB/s) or 46 + 30% (32 heads of 128 x 128, 4096 steps in
// segments of 256: 52 us), and LDS is busy for 40% and 22%.  So the next chunk's rows are loaded
// into registers while this one is computed (barriers order LDS only), the operands of the next
// products are read from LDS while these run, what depends on the thread alone is not computed again
// for every row, and tiles are kept below 80 KiB of LDS, C = 32 instead of 64 where needed, so that
// two blocks share a CU.
#pragma once

#include <type_traits>

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

// x + decay S.  S 2^exponent is exact, and no further from zero than the product: zero stays zero, and
// nothing overflows that the product does not.
__device__ __forceinline__ float decayed(SegDecay decay, float S, float x) {
    return fmaf(decay.factor, __builtin_amdgcn_ldexpf(S, decay.exponent), x);
}

// 2^total (exponents beyond +-1000 make every float32 infinite or zero, and so do these)
__device__ __forceinline__ SegDecay seg_decay_of(double total) {
    const double whole = floor(total);
    return {__builtin_amdgcn_exp2f((float)(total - whole)), (int)fmin(fmax(whole, -1000.0), 1000.0)};
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

// padded width of the summed side, and columns of the state per block: 128 where they fill more than
// half of them and Kd <= 128, else 64.  A block has four waves of 32 or 16 columns; with float32, whose
// LDS tiles leave room for one or two blocks only, eight of 16 instead of four of 32.
constexpr int kt_of(int Kd) { return Kd <= 32 ? 32 : Kd <= 64 ? 64 : Kd <= 128 ? 128 : 256; }
constexpr int nb_of(int KT, int N) { return N > 64 && KT <= 128 ? 128 : 64; }

// what a walk leaves: the state that each segment adds by itself, from zero, and its decay; the
// outputs (and the last state) from the state entering each segment; and with them the dots and the
// states at the anchors
enum { kStates = 0, kOut = 1, kOutDots = 2 };

template <int NPI, int KT, int NW, int CT, int MODE>   // waves, 16-column tiles per wave
struct LinTile {
    static constexpr bool OUT = MODE != kStates;
    static constexpr int NB = 16 * NW * CT, TH = 64 * NW;
    // LDS row pitches, in which neither rows read 8 or 4 elements a lane nor rows read across meet in
    // a bank (for 4 elements a lane: with k's columns of each 16 swapped by halves in rows 8..15 of 16).
    // Conflicts still take 9 to 21% of the LDS cycles of walks with outputs (14% with 32 heads of 64 x 64,
    // 65536 steps, 21% with heads of 128 x 128) and none to 9% of those without; with KT + 8 for q, k as it is, and the scores' tiles
    // stored apart, they took 38% and the walk 8% longer.
    static constexpr int PQ = KT + 16, PK = KT + 16, PV = NB + 16;
    static constexpr int pairs(int C) { return C == 64 ? 6 : 2; }   // (16 outputs, 32 sources) not all above the diagonal
    static constexpr int bytes(int C) {
        return NPI * C * 2 * ((OUT ? PQ : 0) + PK + PV) + (OUT ? pairs(C) * 3 * 1024 : 0) + 2 * (4 * C + 4) * 4 +
               (MODE == kOutDots ? NW * C * 4 : 0);
    }
    static constexpr int C = bytes(64) <= 80 * 1024 ? 64 : 32;
    static constexpr int lds = bytes(C);
    static constexpr int fit = 160 * 1024 / lds * NW / 4;
    static constexpr int most = KT == 256 || (CT == 2 && (OUT || KT == 128)) ? 2 : CT == 2 ? 3 : 4;   // (registers)
    static constexpr int waves = fit > most ? most : fit;           // per SIMD
};

struct LinRoles {
    LinRole r[3];
};

template <int KT_, int NW_, int CT_>
struct WalkShape {
    static constexpr int KT = KT_, NW = NW_, CT = CT_;
};

// f(WalkShape) of operands of NPI parts; narrow: 64 columns a block however many there are
template <int NPI, class Fn>
int with_walk_shape(int Kd, int N, bool narrow, Fn f) {
    const int KT = kt_of(Kd);
    if (KT == 256) return f(WalkShape<256, 4, 1>{});
    if (narrow || nb_of(KT, N) == 64) {
        if (KT == 32) return f(WalkShape<32, 4, 1>{});
        if (KT == 64) return f(WalkShape<64, 4, 1>{});
        return f(WalkShape<128, 4, 1>{});
    }
    constexpr int NW = NPI == 3 ? 8 : 4, CT = 8 / NW;
    if (KT == 32) return f(WalkShape<32, NW, CT>{});
    if (KT == 64) return f(WalkShape<64, NW, CT>{});
    return f(WalkShape<128, NW, CT>{});
}

// ---- loads of a chunk's rows -----------------------------------------------------------------

typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef short v4s __attribute__((ext_vector_type(4)));

// x again, as a value that the compiler does not know to be the same: what is computed from it stays
// where it is written, instead of living in registers across the walk's loop
__device__ __forceinline__ int afresh(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// Offsets of 2^31 or more lie outside every resource used here: loads give zero, stores are dropped.
// (A resource spans C rows of at most 2^24 bytes, 2^30; an offset outside that is moved by less than
// 2^30 either way still lies beyond it.)
constexpr uint32_t kOutside = 0x80000000u;

// One operand's rows of one (sequence, head): W columns from col0 on, C rows a chunk, NU units of 16
// bytes a thread.  A chunk is read as a bounded buffer, whose 32-bit offsets (C st stays below 2^31
// bytes by the limit on st) are the same for every chunk: by units where rows start on 16 bytes and
// do not overlap, rows behind the sequence's end then lying outside; else by elements.
template <class Ty, int C, int W, int TH>
struct RowTile {
    using T = typename Ty::T;
    static constexpr int E = 16 / sizeof(T), UPR = W / E, NU = (C * UPR + TH - 1) / TH, ROWS = TH / UPR;
    const char *base;              // of the next chunk
    int st, col0, width, step;     // st, step in bytes
    uint32_t off;                  // of the first unit
    bool fast, rev;
    v4u u[NU];

    __device__ __forceinline__ void init(const LinView &x, int b, int h, int col0_, int width_, bool rev_, int t0) {
        base = (const char *)((const T *)x.p + b * x.sb + (h / x.r) * x.sh + t0 * x.st);
        st = (int)(x.st * (long)sizeof(T)), col0 = col0_, width = width_, rev = rev_;
        step = rev ? -ROWS * st : ROWS * st;
        const int row = threadIdx.x / UPR, d = col0 + threadIdx.x % UPR * E;
        off = d < width && row < C ? (uint32_t)((rev ? C - 1 - row : row) * st + d * (int)sizeof(T)) : kOutside;
        fast = (((uintptr_t)base | (uintptr_t)st) & 15) == 0 && width % E == 0 && x.st >= width;
    }

    __device__ __forceinline__ void load(int rows) {           // rows: how many exist, any number below 1 for none
        const auto rs = bounded_rsrc(base, rows > 0 ? (uint32_t)((rows - 1) * st + width * (int)sizeof(T)) : 0u);
        base += (long)(rev ? -C : C) * st;
        const uint32_t o = (uint32_t)afresh((int)off);
        if (fast) {
#pragma unroll
            for (int i = 0; i < NU; ++i)
                u[i] = __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)(o + (uint32_t)(i * step)), 0, 0));
            return;
        }
        const int tid = afresh((int)threadIdx.x), d = col0 + tid % UPR * E;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int row = i * ROWS + tid / UPR, j = rev ? C - 1 - row : row;
            const bool on = row < C && j < rows;
            uint32_t x[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const uint32_t at = on && d + e < width ? o + (uint32_t)(i * step + e * (int)sizeof(T)) : kOutside;
                if constexpr (sizeof(T) == 4) x[e] = bload_u(rs, at, 0);
                else x[e] = __builtin_bit_cast(uint16_t, __builtin_amdgcn_raw_buffer_load_b16(rs, (int)at, 0, 0));
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) u[i][k] = sizeof(T) == 4 ? x[k] : x[2 * k] | x[2 * k + 1] << 16;
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    // planes of bf16 parts [C][pitch]; PERM: the columns of each 32 in the order 4 g + 0..3, 16 + 4 g + 0..3;
    // SWAP: the columns of each 16 swapped by halves in every other eight rows
    template <bool PERM, bool SWAP>
    __device__ __forceinline__ void store(uint16_t *lds, const int pitch) const {
        constexpr int NP = InParts<Ty>::n;
        static_assert(TH % UPR == 0 && (ROWS & (ROWS - 1)) == 0, "");
        // everything that depends on the thread stands outside the loop: its units are ROWS rows apart
        const uint32_t tid = (uint32_t)afresh((int)threadIdx.x), row0 = tid / UPR, d = tid % UPR * E;
        const uint32_t swap0 = SWAP ? row0 & 8 : 0;
        lds += row0 * pitch;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            if (C * UPR % TH != 0 && i * ROWS + row0 >= C) continue;
            const uint32_t swap = SWAP ? swap0 ^ (i * ROWS & 8) : 0;
            if constexpr (NP == 1 && !PERM) {
                *(v4u *)(lds + i * ROWS * pitch + (d ^ swap)) = u[i];
                continue;
            }
#pragma unroll
            for (int half = 0; half < E / 4; ++half) {   // four elements at a time
                uint32_t p[NP][2];
                parts(u[i], half, p);
                const uint32_t e = d + 4 * half;
                const uint32_t at = PERM ? (e & ~31) + ((e & 15) >> 2) * 8 + ((e >> 4) & 1) * 4 : e ^ swap;
#pragma unroll
                for (int q = 0; q < NP; ++q)
                    *(v2u *)(lds + (q * C + i * ROWS) * pitch + at) = v2u{p[q][0], p[q][1]};
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

// LDS rows read across: each group of 16 lanes (4 rows x 4 lanes, lane 4 i + j at columns 4 j + 0..3 of
// row i, p its own address) gets 16 columns, lane c the four rows' elements of column c
__device__ __forceinline__ v2u read_turned(const uint16_t *p) {
    return __builtin_bit_cast(
        v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)p));
}

// the three parts of eight floats, as one operand each
__device__ __forceinline__ void split8(const float (&x)[8], v4u (&p)[3]) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t s[3];
        split_pair(x[2 * w], x[2 * w + 1], s);
#pragma unroll
        for (int q = 0; q < 3; ++q) p[q][w] = s[q];
    }
}

// acc += sum of the products of parts whose indices add up to at most 2, the smallest first: all of
// operands of one and two parts, and of three parts all but those below 2^-23 of the whole
template <int NA, int NB>
__device__ __forceinline__ v4f mfma_parts(const v4u (&x)[NA], const v4u (&y)[NB], v4f acc) {
#pragma unroll
    for (int s = 2; s >= 0; --s)
#pragma unroll
        for (int p = 0; p < NA; ++p) {
            const int q = s - p;
            if (q >= 0 && q < NB) acc = mfma_b(x[p], y[q], acc);
        }
    return acc;
}

// the same of every pair of X and Y operands, acc(x, y) += x y, so that consecutive products
// belong to different sums
template <int X, int Y, int NA, int NB, class Acc>
__device__ __forceinline__ void mfma_block(const v4u (&x)[X][NA], const v4u (&y)[Y][NB], Acc acc) {
#pragma unroll
    for (int s = 2; s >= 0; --s)
#pragma unroll
        for (int p = 0; p < NA; ++p) {
            const int q = s - p;
            if (q < 0 || q >= NB) continue;
#pragma unroll
            for (int i = 0; i < X; ++i)
#pragma unroll
                for (int j = 0; j < Y; ++j) acc(i, j) = mfma_b(x[i][p], y[j][q], acc(i, j));
        }
}

// ---- decays of a chunk --------------------------------------------------------------------------

template <int C>
struct Decays {
    float hi[C], lo[C];   // log2 decay summed up to each step
    float into[C];        // sc_kv exp2(L - c - ls'): what a step's k v^T has left at the chunk's end
    float from[C];        // sc_o exp2(c + ls): what the registers' state has left at each step
    float all;            // power of two that the registers take at the chunk's end
    float before, after;  // exp2(ls), exp2(ls'): the state is this times the registers
    float pad;
};
// The registers hold the state up to a factor 2^ls with |ls| <= 1/2, kept in float64 by the last wave.
// So a chunk's decay multiplies them by a power of two, which rounds nothing: rounded to float32, the
// same decay in every chunk would be off the same way each time, by 2^-25 for each of the chunks that a
// state lasts.  (Leaving powers of up to 2^24 in ls as well would save 0 to 4% of the time and cost 24
// bits of the state's range.)

// the double that the DPP control CTRL brings from another lane, 0 where it brings none
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_or_zero(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t l = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 15, false);
    const uint32_t h = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 15, false);
    return __builtin_bit_cast(double, ((uint64_t)h << 32) | l);
}

// by one wave; raw: this lane's log decay (C = 32: the upper half wave repeats the lower), ls: of the
// registers, before and after the chunk.  Returns L.
template <int C>
__device__ __forceinline__ double chunk_decays(Decays<C> &d, float raw, float sc_kv, float sc_o, double &ls) {
    const int lane = threadIdx.x & 63, i = lane & (C - 1);
    double s = gate_of(raw);
    s += dpp_or_zero<0x111, 15>(s);        // row_shr: lanes of each 16
    s += dpp_or_zero<0x112, 15>(s);
    s += dpp_or_zero<0x114, 15>(s);
    s += dpp_or_zero<0x118, 15>(s);
    s += dpp_or_zero<0x142, 0xa>(s);       // row_bcast:15 into rows 1 and 3
    if (C == 64) s += dpp_or_zero<0x143, 0xc>(s);   // row_bcast:31 into rows 2 and 3
    const uint64_t u = __builtin_bit_cast(uint64_t, s);
    const double L = __builtin_bit_cast(
        double, ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), C - 1) << 32) |
                    (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, C - 1));
    const float hi = (float)s;
    d.hi[i] = hi;
    d.lo[i] = (float)(s - (double)hi);
    d.from[i] = sc_o * __builtin_amdgcn_exp2f((float)(s + ls));
    const double next = ls + L, whole = __builtin_rint(next);
    d.into[i] = sc_kv * __builtin_amdgcn_exp2f((float)(whole - (s + ls)));
    if (i == 0) {
        d.before = __builtin_amdgcn_exp2f((float)ls);
        d.all = __builtin_amdgcn_ldexpf(1.f, (int)whole);
        d.after = __builtin_amdgcn_exp2f((float)(next - whole));
    }
    ls = next - whole;
    return L;
}

// ---- the walk ---------------------------------------------------------------------------------

template <class Ty, int KT, int NW, int CT, int MODE>
__global__ __launch_bounds__(64 * NW, (LinTile<InParts<Ty>::n, KT, NW, CT, MODE>::waves)) void k_lin_walk(LinArgs a,
                                                                                                         LinRoles rs) {
    constexpr int NPI = InParts<Ty>::n;
    using Tile = LinTile<NPI, KT, NW, CT, MODE>;
    using T = typename Ty::T;
    constexpr bool OUT = Tile::OUT, DOTS = MODE == kOutDots;
    constexpr int C = Tile::C, NB = Tile::NB, TH = Tile::TH, PQ = Tile::PQ, PK = Tile::PK, PV = Tile::PV;
    constexpr int NT = C / 16, KS = C / 32, DT = KT / 16;
    // operands read from LDS at a time: as many as the registers hold twice (dividing KT / 32, NT, DT)
    constexpr bool TIGHT = KT == 128 && Tile::waves == 4;
    constexpr int UB = TIGHT || NPI == 3 || KT == 32 ? 1 : 2;
    constexpr int QB = TIGHT || CT == 2 || KT == 256 ? 2 : NT, KB = NPI == 1 && !TIGHT && DT > 2 ? 4 : 2;
    extern __shared__ __align__(16) unsigned char smem[];
    uint16_t *Ks = (uint16_t *)smem, *Vs = Ks + NPI * C * PK, *Qs = Vs + NPI * C * PV;
    unsigned char *rest = (unsigned char *)(Qs + (OUT ? NPI * C * PQ : 0));
    constexpr int PAIRS = Tile::pairs(C);
    v4u *Ps = (v4u *)rest;                                     // [PAIRS][3][64 lanes]
    auto pair = [](int it, int ks) { return it < 2 ? it : 2 * it - 2 + ks; };
    Decays<C> *dec = (Decays<C> *)(rest + (OUT ? PAIRS * 3 * 1024 : 0));
    float *dots = (float *)(dec + 2);                          // [NW][C]

    const LinRole ro = rs.r[blockIdx.y];
    const int tiles = (ro.N + NB - 1) / NB;
    const long units = (long)a.B * a.H * a.nseg * tiles;
    if ((long)blockIdx.x >= units) return;
    const int tile = blockIdx.x % tiles, seg = blockIdx.x / tiles % a.nseg, bh = blockIdx.x / tiles / a.nseg;
    const int b = bh / a.H, h = bh % a.H;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // the lane, found anew in each phase: what depends on it takes no registers in the others
    auto lane_now = [] { return afresh((int)threadIdx.x) & 63; };
    const bool rev = ro.reverse;
    const int len = length_of(a, b);
    const int lo = seg * a.seg_steps, hi = lo + a.seg_steps < a.T ? lo + a.seg_steps : a.T;
    const int chunks = (hi - lo + C - 1) / C;
    const int Kd = ro.Kd, N = ro.N;
    const size_t mat = (size_t)Kd * N;
    const int col0 = tile * NB, n0 = col0 + w * 16 * CT;       // the block's and the wave's first column

    const bool last = seg == (rev ? 0 : a.nseg - 1);           // in the walk's order
    if (!OUT && last) return;                                  // adds to no other

    auto t0_of = [&](int n) { return lo + (rev ? chunks - 1 - n : n) * C; };
    RowTile<Ty, C, KT, TH> qr, kr;
    RowTile<Ty, C, NB, TH> vr;
    kr.init(ro.k, b, h, 0, Kd, rev, t0_of(0));
    vr.init(ro.v, b, h, col0, N, rev, t0_of(0));
    if constexpr (OUT) qr.init(ro.q, b, h, 0, Kd, rev, t0_of(0));
    auto rows_of = [&](int n) { return len - t0_of(n) < C ? len - t0_of(n) : C; };
    auto gate = [&](int n) {
        if (n >= chunks) return 0.f;
        const int i = threadIdx.x & (C - 1);
        return gate_raw(a, b, h, t0_of(n) + (rev ? C - 1 - i : i), len, rev);
    };

    kr.load(rows_of(0));
    vr.load(rows_of(0));
    if constexpr (OUT) qr.load(rows_of(0));
    // Column c of the wave's tile ct is column n0 + col(c, ct): with two tiles a lane's four outputs
    // of both are eight columns in a row.
    auto col = [](int c, int ct) { return CT == 2 ? 8 * (c >> 2) + 4 * ct + (c & 3) : c; };
    // element (d, n) of a matrix of Kd N floats, beyond its rows and columns outside
    v4f S[DT][CT];
    auto at = [&](int l, int dt, int ct, int r, int sd, int sn) {
        const int d = dt * 16 + 4 * (l >> 4) + r, n = n0 + col(l & 15, ct);
        return d < Kd && n < N ? (uint32_t)(d * sd + n * sn) * 4u : kOutside;
    };
    {
        const int l = threadIdx.x & 63;
        auto add_to = [&](SegDecay f, const float *src, int sd, int sn) {   // S = f S + src
            const auto rsrc = bounded_rsrc(src, src ? (uint32_t)(mat * 4) : 0u);
            v4f x[DT][CT];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[dt][ct][r] = bload(rsrc, at(l, dt, ct, r, sd, sn), 0);
            __builtin_amdgcn_sched_barrier(0);                 // (all loads in flight before the first is used)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int r = 0; r < 4; ++r) S[dt][ct][r] = decayed(f, S[dt][ct][r], x[dt][ct][r]);
        };
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) S[dt][ct] = v4f{0.f, 0.f, 0.f, 0.f};
        if constexpr (OUT) {
            const float *own = ro.seg + ((size_t)bh * a.nseg + seg) * mat;
            if (a.joined) add_to({0.f, 0}, own, ro.seg_d, ro.seg_n);
            else add_to({0.f, 0}, ro.init ? ro.init + bh * mat : nullptr, ro.init_d, ro.init_n);
            if (!a.joined)                                     // the segments before this one
                for (int s = rev ? a.nseg - 1 : 0; s != seg; s += rev ? -1 : 1)
                    add_to(ro.seg_decay[(size_t)bh * a.nseg + s], own + ((long)s - seg) * (long)mat, ro.seg_d, ro.seg_n);
        }
    }
    auto put_state = [&](float *dst, int sd, int sn, float f) {
        const auto rsrc = bounded_rsrc(dst, (uint32_t)(mat * 4));
        const int l = afresh((int)threadIdx.x) & 63;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    bstore_u(rsrc, __float_as_uint(f * S[dt][ct][r]), at(l, dt, ct, r, sd, sn), 0);
                    if (r == 3) __builtin_amdgcn_sched_barrier(0);
                }
    };

    // this lane's part of the outputs: step i = 16 it + c of a chunk, columns n0 + 4 CT g + 0 .. 4 CT - 1
    const int out_size = ro.out_f32 ? 4 : (int)sizeof(T), out_row = a.H * N * out_size;   // C rows below 2^31 bytes
    auto out_off = [&](int l, int row, int size) {             // of it = 0; the others 16 rows further each
        const int n = n0 + 4 * CT * (l >> 4);
        return n < N ? (uint32_t)((rev ? C - 1 - (l & 15) : l & 15) * row + n * size) : kOutside;
    };
    const T *partner = nullptr;
    bool partner_fast = false;
    const bool dotted = DOTS && ro.dot;                        // (dv's role, beside those of dq and dk, has none)
    if (dotted) {
        partner = (const T *)ro.partner.p + b * ro.partner.sb + (h / ro.partner.r) * ro.partner.sh;
        const long row = ro.partner.st * (long)sizeof(T);
        partner_fast = (((uintptr_t)partner | (uintptr_t)row) & (4 * CT * sizeof(T) - 1) & 15) == 0 && N % (4 * CT) == 0 &&
                       ro.partner.st >= N;
    }

    // the tile above the diagonal that shares an operand with the first stays zero
    if constexpr (OUT && C == 32)
        for (int i = threadIdx.x; i < PAIRS * 3 * 64; i += TH) Ps[i] = v4u{0, 0, 0, 0};
    auto store = [&] {
        kr.template store<false, OUT>(Ks, PK);
        vr.template store<false, false>(Vs, PV);
        if constexpr (OUT) qr.template store<true, false>(Qs, PQ);
    };
    double total = 0.0, ls = 0.0;                              // last wave: log2 decay of the segment, the registers' scale
    float raw = 0.f;
    if (w == NW - 1) {
        const double L = chunk_decays<C>(dec[0], gate(0), ro.sc_kv, ro.sc_o, ls);
        if (!OUT) total += L;
        raw = __int_as_float(afresh(__float_as_int(gate(1))));
    }
    const int na = (a.T + kLinAnchor - 1) / kLinAnchor;
    const float sc_p = ro.sc_kv * ro.sc_o;
    const bool keep = ro.fin && last;                          // the state behind the last step is wanted
    store();

    // The next chunk's rows are loaded while this one is computed and go to LDS before this one's
    // results go out: the wait for loads is then never one for stores too.
    for (int n = 0; n < chunks; ++n) {
        const int t0 = t0_of(n);
        const Decays<C> &dc = dec[n & 1];
        lds_barrier();
        const bool ahead = n + 1 < chunks;
        const int rows_ahead = rows_of(n + 1);
        if (ahead) {                    // (v's and q's rows follow between the products)
            const float next = raw;
            if (w == NW - 1) raw = gate(n + 2);
            kr.load(rows_ahead);
            if (!OUT) vr.load(rows_ahead);
            if (w == NW - 1) {
                const double L = chunk_decays<C>(dec[(n + 1) & 1], next, ro.sc_kv, ro.sc_o, ls);
                if (!OUT) total += L;
            }
        }
        float *anc = nullptr;
        if constexpr (DOTS) {
            if (dotted && ((t0 + C) % kLinAnchor == 0 || t0 + C >= a.T)) anc = ro.anchor + ((size_t)bh * na + t0 / kLinAnchor) * mat;
            if (anc && rev) put_state(anc, N, 1, dc.before);
        }
        __builtin_amdgcn_sched_barrier(0);

        v4f O[NT][CT];
        if constexpr (OUT) {
            // decayed scores, transposed (rows j, columns i), in tiles of those on and below the diagonal.
            // C = 32: one tile for each of the first three waves.  C = 64: two tiles of one row for each
            // wave, which share its q, and for waves 0 and 1 the first tile of row 2 w.
            constexpr bool TWO = C == 64;
            static_assert(!TWO || NW == 4, "");
            auto scores = [&](auto count) {
                constexpr int M = decltype(count)::value;
                const int lane = lane_now(), g = lane >> 4, c = lane & 15;
                int it[M], jt[M];
                it[0] = TWO ? (w < 3 ? w + 1 : 3) : (w + 1) / 2;
                jt[0] = TWO ? (w < 3 ? 0 : 2) : w / 2;
                if constexpr (M > 1) it[1] = it[0], jt[1] = jt[0] + 1;
                if constexpr (M > 2) it[2] = jt[2] = 2 * w;
                float hi_i[M], lo_i[M];
                v4f hi_j[M], lo_j[M], acc[M];
#pragma unroll
                for (int m = 0; m < M; ++m) acc[m] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int u0 = 0; u0 < KT / 32; u0 += UB) {
                    v4u kf[M][UB][NPI], qf[M][UB][NPI];
#pragma unroll
                    for (int m = 0; m < M; ++m)
#pragma unroll
                        for (int u = 0; u < UB; ++u)
#pragma unroll
                            for (int p = 0; p < NPI; ++p) {
                                const uint16_t *kp = Ks + (p * C + jt[m] * 16 + c) * PK + (u0 + u) * 32 + (4 * g ^ (c & 8));
                                const v2u k0 = *(const v2u *)kp, k1 = *(const v2u *)(kp + 16);
                                kf[m][u][p] = v4u{k0[0], k0[1], k1[0], k1[1]};
                                if (m != 1) qf[m][u][p] = *(const v4u *)(Qs + (p * C + it[m] * 16 + c) * PQ + (u0 + u) * 32 + 8 * g);
                            }
                    if (u0 + UB >= KT / 32)
#pragma unroll
                        for (int m = 0; m < M; ++m) {
                            hi_i[m] = dc.hi[it[m] * 16 + c], lo_i[m] = dc.lo[it[m] * 16 + c];
                            hi_j[m] = *(const v4f *)(dc.hi + jt[m] * 16 + 4 * g);
                            lo_j[m] = *(const v4f *)(dc.lo + jt[m] * 16 + 4 * g);
                        }
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int u = 0; u < UB; ++u)
#pragma unroll
                        for (int m = 0; m < M; ++m) acc[m] = mfma_parts(kf[m][u], qf[m == 1 ? 0 : m][u], acc[m]);
                }
                uint32_t pp[M][2][3];
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    const int above = it[m] == jt[m] ? 4 * g - c : -64;   // j - i of the first row, on the diagonal
                    float x[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float e = (hi_i[m] - hi_j[m][r]) + (lo_i[m] - lo_j[m][r]);
                        const float p = acc[m][r] * sc_p * __builtin_amdgcn_exp2f(e);
                        x[r] = above + r <= 0 ? p : 0.f;
                    }
                    split_pair(x[0], x[1], pp[m][0]);
                    split_pair(x[2], x[3], pp[m][1]);
                }
                auto operand = [&](int m) { return Ps + pair(it[m], jt[m] >> 1) * 3 * 64 + lane; };
#pragma unroll
                for (int q = 0; q < 3; ++q) {
                    if constexpr (TWO) operand(0)[q * 64] = v4u{pp[0][0][q], pp[0][1][q], pp[1][0][q], pp[1][1][q]};
                    else *((v2u *)(operand(0) + q * 64) + (jt[0] & 1)) = v2u{pp[0][0][q], pp[0][1][q]};
                    if constexpr (M > 2) operand(2)[q * 64] = v4u{pp[2][0][q], pp[2][1][q], 0, 0};   // (above the diagonal)
                }
            };
            if constexpr (TWO) {
                if (w < 2) scores(std::integral_constant<int, 3>{});
                else scores(std::integral_constant<int, 2>{});
            } else if (w < 3) {
                scores(std::integral_constant<int, 1>{});
            }
            if (ahead) vr.load(rows_ahead);
            // what the entering state gives, transposed: rows n, columns i
            const int lane = lane_now(), g = lane >> 4, c = lane & 15;
#pragma unroll
            for (int it = 0; it < NT; ++it)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) O[it][ct] = v4f{0.f, 0.f, 0.f, 0.f};
            v4u qf[2][QB][NPI];   // read QB at a time, one time ahead
            auto read_q = [&](int n) {
                const int u = n / (NT / QB), it0 = n % (NT / QB) * QB;
#pragma unroll
                for (int m = 0; m < QB; ++m)
#pragma unroll
                    for (int p = 0; p < NPI; ++p)
                        qf[n & 1][m][p] = *(const v4u *)(Qs + (p * C + (it0 + m) * 16 + c) * PQ + u * 32 + 8 * g);
            };
            constexpr int QN = KT / 32 * (NT / QB);
            read_q(0);
            v4u sf[CT][3];
#pragma unroll
            for (int n = 0; n < QN; ++n) {
                const int u = n / (NT / QB), it0 = n % (NT / QB) * QB;
                if (n + 1 < QN) read_q(n + 1);
                __builtin_amdgcn_sched_barrier(0);
                if (it0 == 0)
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) {
                        float x[8];
#pragma unroll
                        for (int r = 0; r < 4; ++r) x[r] = S[2 * u][ct][r], x[4 + r] = S[2 * u + 1][ct][r];
                        split8(x, sf[ct]);
                    }
                mfma_block<CT, QB>(sf, qf[n & 1], [&](int ct, int m) -> v4f & { return O[it0 + m][ct]; });
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int it = 0; it < NT; ++it) {
                const float f = dc.from[it * 16 + c];
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) O[it][ct] *= f;
            }
            if (ahead) qr.load(rows_ahead);
            lds_barrier();
        }

        constexpr int PW = 4 * CT * sizeof(T) / 4 < 4 ? 1 : CT * sizeof(T) / 4;   // 16-byte words of a partner row
        v4u pr[DOTS ? NT : 1][PW];    // the partner's rows, used at the end
        auto read_partner = [&] {
            const int rows = len - t0 < C ? len - t0 : C;
            const auto prs = bounded_rsrc(partner + t0 * ro.partner.st,
                                          rows > 0 ? (uint32_t)(((rows - 1) * ro.partner.st + N) * sizeof(T)) : 0u);
            const int row = (int)(ro.partner.st * (long)sizeof(T)), l = afresh((int)threadIdx.x) & 63;
            const uint32_t off0 = out_off(l, row, sizeof(T));
#pragma unroll
            for (int it = 0; it < NT; ++it) {
                const uint32_t off = off0 + (uint32_t)((rev ? -16 * it : 16 * it) * row);
                if (partner_fast) {
                    if constexpr (4 * CT * sizeof(T) == 8) {
                        const v2u x = __builtin_bit_cast(v2u, __builtin_amdgcn_raw_buffer_load_b64(prs, (int)off, 0, 0));
                        pr[it][0] = v4u{x[0], x[1], 0, 0};
                    } else {
#pragma unroll
                        for (int k = 0; k < PW; ++k)
                            pr[it][k] = __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(prs, (int)(off + 16 * k), 0, 0));
                    }
                    continue;
                }
                const int i = it * 16 + (l & 15), j = rev ? C - 1 - i : i, nn = n0 + 4 * CT * (l >> 4);
#pragma unroll
                for (int k = 0; k < PW; ++k) pr[it][k] = v4u{0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 4 * CT; ++e) {
                    const uint32_t p = j < rows && nn + e < N ? off + e * (uint32_t)sizeof(T) : kOutside;
                    if constexpr (sizeof(T) == 4)
                        pr[it][e / 4][e % 4] = bload_u(prs, p, 0);
                    else
                        pr[it][e / 8][e / 2 % 4] |= (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(prs, (int)p, 0, 0)
                                                    << (e & 1) * 16;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };

        // the chunk's own steps, and (STATE) the state at its end
        auto finish = [&](auto state) {
        constexpr bool STATE = decltype(state)::value;
        if constexpr (STATE) {
            const float all = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(dc.all)));
            if (all != 1.f)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) S[dt][ct] *= all;
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int lane = lane_now(), g = lane >> 4, c = lane & 15;
            v4u vf[CT][NPI], sv[CT][3];
            const v4f into0 = *(const v4f *)(dc.into + ks * 32 + 4 * g), into1 = *(const v4f *)(dc.into + ks * 32 + 16 + 4 * g);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int p = 0; p < NPI; ++p) {
                    const uint16_t *vp = Vs + p * C * PV + w * 16 * CT + (CT == 2 ? 8 * (c & 3) + 4 * ct : 4 * (c & 3));
                    const v2u v0 = read_turned(vp + (ks * 32 + 4 * g + (c >> 2)) * PV);
                    const v2u v1 = read_turned(vp + (ks * 32 + 16 + 4 * g + (c >> 2)) * PV);
                    vf[ct][p] = v4u{v0[0], v0[1], v1[0], v1[1]};
                }
            v4u pf[2][1][3], kf[2][KB][NPI];   // the operands of the next products read while these run
            auto read_p = [&](int it) {
#pragma unroll
                for (int q = 0; q < 3; ++q) pf[it & 1][0][q] = Ps[(pair(it, ks) * 3 + q) * 64 + lane];
            };
            auto read_k = [&](int n) {
#pragma unroll
                for (int m = 0; m < KB; ++m)
#pragma unroll
                    for (int p = 0; p < NPI; ++p) {
                        const uint16_t *kp = Ks + p * C * PK + (ks * 32 + 4 * g + (c >> 2)) * PK + (n * KB + m) * 16 +
                                             (4 * (c & 3) ^ (OUT ? (g >> 1) * 8 : 0));
                        const v2u k0 = read_turned(kp), k1 = read_turned(kp + 16 * PK);
                        kf[n & 1][m][p] = v4u{k0[0], k0[1], k1[0], k1[1]};
                    }
            };
            if constexpr (OUT) read_p(2 * ks);
            else read_k(0);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (STATE)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                float x[8];
#pragma unroll
                for (int p = 0; p < NPI; ++p)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float x0 = __uint_as_float(vf[ct][p][e] << 16), x1 = __uint_as_float(vf[ct][p][e] & 0xffff0000u);
                        x[2 * e] = p ? x[2 * e] + x0 : x0;
                        x[2 * e + 1] = p ? x[2 * e + 1] + x1 : x1;
                    }
#pragma unroll
                for (int r = 0; r < 4; ++r) x[r] *= into0[r], x[4 + r] *= into1[r];
                split8(x, sv[ct]);
            }
            if constexpr (OUT) {
#pragma unroll
                for (int it = 0; it < NT; ++it) {
                    if (it < 2 * ks) continue;                 // (all of its sources lie above the diagonal)
                    if (it + 1 < NT) read_p(it + 1);
                    else if (STATE) read_k(0);
                    __builtin_amdgcn_sched_barrier(0);
                    mfma_block<CT, 1>(vf, pf[it & 1], [&](int ct, int) -> v4f & { return O[it][ct]; });
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if constexpr (DOTS)
                if (ks == KS - 1 && dotted) read_partner();
            if constexpr (STATE)
#pragma unroll
            for (int n = 0; n < DT / KB; ++n) {
                if (n + 1 < DT / KB) read_k(n + 1);
                __builtin_amdgcn_sched_barrier(0);
                mfma_block<KB, CT>(kf[n & 1], sv, [&](int m, int ct) -> v4f & { return S[n * KB + m][ct]; });
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        };
        if (!OUT || DOTS || ahead || keep) finish(std::true_type{});
        else if constexpr (MODE == kOut) finish(std::false_type{});

        if (dotted) {
            const int lane = lane_now(), g = lane >> 4, c = lane & 15;
#pragma unroll
            for (int it = 0; it < NT; ++it) {
                const int i = it * 16 + c;
                float dot = 0.f;
#pragma unroll
                for (int e = 0; e < 4 * CT; ++e) {
                    float y;
                    if constexpr (sizeof(T) == 4) {
                        y = __uint_as_float(pr[it][e / 4][e % 4]);
                    } else {
                        const uint16_t u = (uint16_t)(pr[it][e / 8][e / 2 % 4] >> (e & 1) * 16);
                        y = Ty::up(__builtin_bit_cast(T, u));
                    }
                    dot = fmaf(O[it][e / 4][e % 4], y, dot);
                }
                dot = group_sum(dot);
                if (g == 0) dots[w * C + i] = t0 + (rev ? C - 1 - i : i) < len ? dot : 0.f;
            }
            if (anc && !rev) put_state(anc, N, 1, dc.after);
        }
        lds_barrier();
        if (ahead) {
            store();
            raw = __int_as_float(afresh(__float_as_int(raw)));   // (loaded before the rows: no wait for it later)
        }
        if constexpr (OUT) {
            const int l = lane_now();
            if (t0 + C > len)             // rows behind the sequence's end: zero
#pragma unroll
                for (int it = 0; it < NT; ++it) {
                    const int i = it * 16 + (l & 15);
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct)
                        if (t0 + (rev ? C - 1 - i : i) >= len) O[it][ct] = v4f{0.f, 0.f, 0.f, 0.f};
                }
            const int rows = a.T - t0 < C ? a.T - t0 : C;
            const size_t first = (((size_t)b * a.T + t0) * a.H + h) * N;
            const auto ors = bounded_rsrc((char *)ro.out + first * out_size,
                                          (uint32_t)((rows - 1) * out_row + N * out_size));
            const uint32_t off0 = out_off(l, out_row, out_size);
            auto off_of = [&](int it) { return off0 + (uint32_t)((rev ? -16 * it : 16 * it) * out_row); };
            if (ro.wide_out && (sizeof(T) == 4 || ro.out_f32)) {
#pragma unroll
                for (int it = 0; it < NT; ++it)
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct)
                        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, O[it][ct]), ors,
                                                               (int)(off_of(it) + ct * 16), 0, 0);
            } else if (ro.wide_out) {
#pragma unroll
                for (int it = 0; it < NT; ++it) {
                    union { T x[4 * CT]; v2u u; v4u v; } y;
#pragma unroll
                    for (int e = 0; e < 4 * CT; ++e) y.x[e] = Ty::down(O[it][e / 4][e % 4]);
                    if constexpr (CT == 2) __builtin_amdgcn_raw_buffer_store_b128(y.v, ors, (int)off_of(it), 0, 0);
                    else __builtin_amdgcn_raw_buffer_store_b64(y.u, ors, (int)off_of(it), 0, 0);
                }
            } else {
                const int nn = n0 + 4 * CT * (l >> 4);
#pragma unroll
                for (int it = 0; it < NT; ++it)
#pragma unroll
                    for (int e = 0; e < 4 * CT; ++e) {
                        const uint32_t p = nn + e < N ? off_of(it) + e * out_size : kOutside;
                        const float o = O[it][e / 4][e % 4];
                        if (sizeof(T) == 4 || ro.out_f32) {
                            bstore_u(ors, __float_as_uint(o), p, 0);
                        } else if constexpr (sizeof(T) == 2) {
                            __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, (T)Ty::down(o)), ors, (int)p, 0, 0);
                        }
                        if (e == 4 * CT - 1) __builtin_amdgcn_sched_barrier(0);
                    }
            }
        }
        if (dotted) {
            const int i = threadIdx.x, t = rev ? t0 + C - 1 - i : t0 + i;
            if (i < C && t < a.T) {
                float d = 0.f;
#pragma unroll
                for (int k = 0; k < NW; ++k) d += dots[k * C + i];
                ro.dot[((size_t)tile * a.B * a.H + bh) * a.T + t] = d;
            }
        }
    }

    if constexpr (OUT) {
        if (keep) {
            const float f = rev ? __builtin_amdgcn_exp2f((float)gate_of(gate_raw(a, b, h, -1, len, true))) : 1.f;
            put_state(ro.fin + bh * mat, ro.fin_d, ro.fin_n, f * dec[(chunks - 1) & 1].after);
        }
    } else {
        put_state(ro.seg + ((size_t)bh * a.nseg + seg) * mat, N, 1, dec[(chunks - 1) & 1].after);
        if (w == NW - 1 && (threadIdx.x & 63) == 0 && tile == 0)
            ro.seg_decay[(size_t)bh * a.nseg + seg] = seg_decay_of(total);
    }
}

// ---- launches -------------------------------------------------------------------------------------

template <class Ty, int KT, int NW, int CT, int MODE>
int launch_walk_tile(const LinArgs &a, const LinRole *roles, int n, hipStream_t st) {
    using Tile = LinTile<InParts<Ty>::n, KT, NW, CT, MODE>;
    LinRoles rs{};
    int tiles = 0;
    for (int i = 0; i < n; ++i) {
        rs.r[i] = roles[i];
        const int t = (roles[i].N + Tile::NB - 1) / Tile::NB;
        tiles = t > tiles ? t : tiles;
    }
    const void *fn = (const void *)k_lin_walk<Ty, KT, NW, CT, MODE>;
    if (Tile::lds > 64 * 1024) DEER_HIP(hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, Tile::lds));
    KTimer kt(MODE == kStates ? "k_lin_walk_states" : "k_lin_walk", st);
    hipLaunchKernelGGL((k_lin_walk<Ty, KT, NW, CT, MODE>), dim3((unsigned)(a.B * a.H * a.nseg * tiles), n),
                       dim3(64 * NW), Tile::lds, st, a, rs);
    DEER_LAUNCH_CHECK("k_lin_walk");
    return DEER_OK;
}

template <class Ty, int MODE>
int launch_walk_mode(const LinArgs &a, const LinRole *roles, int n, hipStream_t st) {
    // Where blocks of 128 columns leave half of the CUs without one, twice as many of 64, which take less
    // time for a chunk (1 x 2048 steps, 4 heads of 128 x 128 in bf16: 34 us, narrow 28; with 256 blocks the
    // second reading of q and k costs more: 8 x 128 steps, 32 heads: 20.6, narrow 22.4).  Not with dots,
    // which are laid out by blocks of 128.
    const int nb = nb_of(kt_of(roles[0].Kd), roles[0].N), tiles = (roles[0].N + nb - 1) / nb;
    const bool narrow = MODE != kOutDots && nb == 128 && (long)a.B * a.H * a.nseg * tiles * n <= 128;
    return with_walk_shape<InParts<Ty>::n>(roles[0].Kd, roles[0].N, narrow, [&](auto s) {
        return launch_walk_tile<Ty, s.KT, s.NW, s.CT, MODE>(a, roles, n, st);
    });
}

template <class Ty>
int launch_walk_type(const LinArgs &a, const LinRole *roles, int n, bool states, bool dots, hipStream_t st) {
    if (states) return launch_walk_mode<Ty, kStates>(a, roles, n, st);
    return dots ? launch_walk_mode<Ty, kOutDots>(a, roles, n, st) : launch_walk_mode<Ty, kOut>(a, roles, n, st);
}

}  // namespace deer
