// C ABI of the layers: linear attention with decays and layer normalisation (argument checks,
// workspace, the operands of each walk).  All device work is queued on the caller's stream.
#include <math.h>
#include <stdlib.h>

#include "common.h"
#include "launch.h"
#include "types16.h"

namespace deer {

static int check_shape(const deer_linattn_shape *s, int B, int T) {
    if (!s) { set_error("shape pointer is NULL"); return DEER_ERR_INVALID_ARG; }
    if (!dtype_ok(s->dtype)) { set_error("unknown dtype %d", s->dtype); return DEER_ERR_INVALID_ARG; }
    if (B <= 0 || T <= 0) { set_error("B and T must be positive (B=%d, T=%d)", B, T); return DEER_ERR_INVALID_ARG; }
    if (s->H <= 0 || s->H > 16384 || s->Hk <= 0 || s->H % s->Hk != 0) {
        set_error("H must be a multiple of Hk in 1..16384 (H=%d, Hk=%d)", s->H, s->Hk);
        return DEER_ERR_INVALID_ARG;
    }
    if (s->Dk < 1 || s->Dk > 256 || s->Dv < 1 || s->Dv > 256) {
        set_error("Dk and Dv must lie in 1..256 (Dk=%d, Dv=%d)", s->Dk, s->Dv);
        return DEER_ERR_INVALID_ARG;
    }
    if (!isfinite(s->scale)) { set_error("scale must be finite"); return DEER_ERR_INVALID_ARG; }
    if ((long)B * s->H > (1L << 20)) { set_error("B H must not exceed 2^20 (B=%d, H=%d)", B, s->H); return DEER_ERR_INVALID_ARG; }
    if (T > (1 << 30) || (double)B * T * s->H > 8589934592.0) {
        set_error("T must not exceed 2^30, nor B T H 2^33 (B=%d, T=%d, H=%d)", B, T, s->H);
        return DEER_ERR_INVALID_ARG;
    }
    return DEER_OK;
}

static int check_view(const deer_view *x, const char *name, int T) {
    if (!x || !x->p) { set_error("%s is required", name); return DEER_ERR_INVALID_ARG; }
    if (x->sb < 0 || x->st < 0 || x->sh < 0) { set_error("the strides of %s must not be negative", name); return DEER_ERR_INVALID_ARG; }
    if (T > 1 && x->st > (1L << 22)) {
        set_error("the step stride of %s must not exceed 2^22 elements", name);
        return DEER_ERR_INVALID_ARG;
    }
    return DEER_OK;
}

// an output that is one of the inputs
static int check_alias(const void *out, const char *name, const void *const *in, int n) {
    for (int i = 0; i < n; ++i)
        if (out && out == in[i]) { set_error("%s may not be an input's memory", name); return DEER_ERR_INVALID_ARG; }
    return DEER_OK;
}

// (a single step's stride says nothing: one that leaves its rows aligned and apart)
static LinView view_of(const deer_view *x, int r, int T) {
    return {x->p, (long)x->sb, T > 1 ? (long)x->st : 256, (long)x->sh, r};
}

// DEER_LIN_SEG=n: segments of n steps (rounded up to 64), whatever the sizes (a tuning and test
// override)
static int seg_override() {
    const char *e = getenv("DEER_LIN_SEG");
    return e ? atoi(e) : 0;
}

// Segments: as many as leave all blocks of a walk resident on the chip at once (a few blocks more
// would run after the others, alone), none of fewer than kMinSeg steps; one where the heads alone give
// half of that, since segments read k and v a second time.  (2 x 4096 steps, 16 heads of 128 x 128 in
// bf16, where one segment gives 32 blocks of 512: segments of 256, 512, 1024, 4096 steps take 85, 87,
// 102, 241 us.)  An adjoint's are sized for two of its three roles, the third's blocks following as others
// end (4 x 4096 steps, 16 heads: segments of 512, 1024, 2048 steps 362, 327, 349 us; the rule takes 1024,
// for three roles it would take 2048).
constexpr int kMinSeg = 128;

static int segment_steps(const deer_linattn_shape *s, int B, int T, int op) {
    if (const int n = seg_override(); n > 0) return n >= T ? T : (n + 63) / 64 * 64;
    const bool adj = op == DEER_OP_ADJOINT;
    const int Kd = adj ? s->Dv : s->Dk, N = adj ? s->Dk : s->Dv;
    const long blocks = (long)B * s->H * lin_tiles(Kd, N) * (adj ? 2 : 1);
    const long fill = 256L * lin_resident(s->dtype, Kd, N, adj);
    if (2 * blocks > fill || T <= kMinSeg) return T;
    const long n = fill / blocks;
    const long steps = ((T + n - 1) / n + 63) / 64 * 64;
    return (int)(steps < kMinSeg ? kMinSeg : steps);
}

// Up to this many segments, a walk's block adds up the states before its own segment by itself,
// beyond that k_lin_join does it once for all (in bf16, 4 segments: 8 x 512 steps of 16 heads of 64 x 64
// forwards 29.0 us, joined 29.4, the adjoint of 4 x 4096 steps of 16 heads of 128 x 128 327, joined 329;
// 2 x 4096 steps of those forwards: 8 segments 90, joined 85; 16 segments 101, joined 80).
constexpr int kMostUnjoined = 4;

static LinArgs args_of(const deer_linattn_shape *s, int B, int T, int op, const float *log_decay,
                       const int32_t *lengths) {
    const int steps = segment_steps(s, B, T, op);
    return {s->dtype, B, T, s->H, log_decay, s->per_step != 0, lengths, steps, (T + steps - 1) / steps, false};
}

struct LinWs {
    float *dq, *dk;              // per head, before the sum over the heads that share them
    float *dq_dot, *dk_dot;      // [tiles][B, H, T]
    float *fwd, *rev;            // states at the anchors [B, H, anchors][Dv, Dk]
    double *part;                // [B, H, anchors]
    float *seg, *rseg;           // [B, H, segments] of the forward state (the adjoint: S^T), and of R
    SegDecay *seg_decay, *rseg_decay;
    size_t bytes;
};

static LinWs carve_lin(void *ws, const deer_linattn_shape *s, int B, int T, int op) {
    LinWs w{};
    Carver c(ws);
    c.take<char>(1);             // a valid query is never zero
    if (op == DEER_OP_ADJOINT) {
        const size_t bh = (size_t)B * s->H, na = (T + kLinAnchor - 1) / kLinAnchor;
        if (s->H != s->Hk) {
            w.dq = c.take<float>(bh * T * s->Dk);
            w.dk = c.take<float>(bh * T * s->Dk);
        }
        const int tiles = lin_tiles(s->Dv, s->Dk);
        w.dq_dot = c.take<float>(tiles * bh * T);
        w.dk_dot = c.take<float>(tiles * bh * T);
        w.fwd = c.take<float>(bh * na * s->Dk * s->Dv);
        w.rev = c.take<float>(bh * na * s->Dk * s->Dv);
        w.part = c.take<double>(bh * na);
    }
    const int steps = segment_steps(s, B, T, op);
    if (steps < T) {
        const size_t n = (size_t)B * s->H * ((T + steps - 1) / steps);
        w.seg = c.take<float>(n * s->Dk * s->Dv);
        w.seg_decay = c.take<SegDecay>(n);
        if (op == DEER_OP_ADJOINT) {
            w.rseg = c.take<float>(n * s->Dk * s->Dv);
            w.rseg_decay = c.take<SegDecay>(n);
        }
    }
    w.bytes = c.off;
    return w;
}

// whether out's rows of N take 16-byte stores of eight elements (or two of four)
static bool wide_out(const void *p, int N) { return N % 8 == 0 && ((uintptr_t)p & 15) == 0; }

static int check_norm(const deer_norm *n, int64_t rows) {
    if (!n) { set_error("norm pointer is NULL"); return DEER_ERR_INVALID_ARG; }
    if (!dtype_ok(n->dtype) || (n->wtype != DEER_F32 && n->wtype != n->dtype)) {
        set_error("unknown types (dtype=%d, wtype=%d: DEER_F32 or dtype)", n->dtype, n->wtype);
        return DEER_ERR_INVALID_ARG;
    }
    if (n->D < 1 || n->D > 65536) { set_error("D must lie in 1..65536 (D=%d)", n->D); return DEER_ERR_INVALID_ARG; }
    if (n->G < 1 || rows < 1 || rows % n->G != 0) {
        set_error("rows must be a positive multiple of G (rows=%lld, G=%d)", (long long)rows, n->G);
        return DEER_ERR_INVALID_ARG;
    }
    if (n->G > (1 << 20) || (long)n->G * n->D > (1L << 24)) {
        set_error("G must not exceed 2^20, nor G D 2^24 (G=%d, D=%d)", n->G, n->D);
        return DEER_ERR_INVALID_ARG;
    }
    if (!(n->eps >= 0.f) || !isfinite(n->eps)) { set_error("eps must be finite and not negative"); return DEER_ERR_INVALID_ARG; }
    return DEER_OK;
}

static NormArgs norm_of(const deer_norm *n, int64_t rows, const void *x) {
    return {n->dtype, n->wtype, (size_t)rows, n->G, n->D, x, n->w, n->b, n->eps};
}

}  // namespace deer

using namespace deer;

extern "C" {

size_t deer_linattn_workspace_bytes(const deer_linattn_shape *s, int B, int T, int op) {
    if (check_shape(s, B, T) != DEER_OK || (op != DEER_OP_SOLVE && op != DEER_OP_ADJOINT)) return 0;
    return carve_lin(nullptr, s, B, T, op).bytes;
}

int deer_linattn(const deer_linattn_shape *s, int B, int T, const deer_view *q, const deer_view *k, const deer_view *v,
                 const float *log_decay, const int32_t *lengths, const float *state0, void *o, float *state, void *ws,
                 size_t ws_bytes, void *stream) {
    set_error("");
    int rc = check_shape(s, B, T);
    if (rc) return rc;
    if ((rc = check_view(q, "q", T)) || (rc = check_view(k, "k", T)) || (rc = check_view(v, "v", T))) return rc;
    if (!log_decay || !o) { set_error("log_decay and o are required"); return DEER_ERR_INVALID_ARG; }
    const void *in[] = {q->p, k->p, v->p, log_decay, state0};
    if ((rc = check_alias(o, "o", in, 5)) || (rc = check_alias(state, "state", in, 4))) return rc;
    if (state && (void *)state == o) { set_error("o and state may not be the same memory"); return DEER_ERR_INVALID_ARG; }
    if ((rc = check_ws(ws, ws_bytes, carve_lin(nullptr, s, B, T, DEER_OP_SOLVE).bytes))) return rc;
    const LinWs w = carve_lin(ws, s, B, T, DEER_OP_SOLVE);
    LinArgs a = args_of(s, B, T, DEER_OP_SOLVE, log_decay, lengths);
    hipStream_t st = (hipStream_t)stream;
    const int r = s->H / s->Hk;
    LinRole ro{};
    ro.q = view_of(q, r, T), ro.k = view_of(k, r, T), ro.v = view_of(v, 1, T);
    ro.Kd = s->Dk, ro.N = s->Dv;
    ro.sc_kv = 1.f, ro.sc_o = s->scale;
    ro.out = o, ro.wide_out = wide_out(o, s->Dv);
    ro.init = state0, ro.init_d = s->Dv, ro.init_n = 1;
    ro.fin = state, ro.fin_d = s->Dv, ro.fin_n = 1;
    if (a.nseg > 1) {
        ro.seg = w.seg, ro.seg_decay = w.seg_decay, ro.seg_d = s->Dv, ro.seg_n = 1;
        if ((rc = launch_lin_walk(a, &ro, 1, true, false, st))) return rc;
        // (state0 updated in place: the last segment's block may not write it while others read it)
        a.joined = a.nseg > kMostUnjoined || (state0 && state == state0);
        if (a.joined && (rc = launch_lin_join(a, &ro, 1, st))) return rc;
    }
    return launch_lin_walk(a, &ro, 1, false, false, st);
}

int deer_linattn_adjoint(const deer_linattn_shape *s, int B, int T, const deer_view *q, const deer_view *k,
                         const deer_view *v, const float *log_decay, const int32_t *lengths, const float *state0,
                         const deer_view *g, const float *g_state, void *dq, void *dk, void *dv, float *dlog_decay,
                         float *dstate0, void *ws, size_t ws_bytes, void *stream) {
    set_error("");
    int rc = check_shape(s, B, T);
    if (rc) return rc;
    if ((rc = check_view(q, "q", T)) || (rc = check_view(k, "k", T)) || (rc = check_view(v, "v", T)) ||
        (rc = check_view(g, "g", T)))
        return rc;
    if (!log_decay || !dq || !dk || !dv) { set_error("log_decay, dq, dk and dv are required"); return DEER_ERR_INVALID_ARG; }
    const void *in[] = {q->p, k->p, v->p, g->p, log_decay, state0, g_state};
    const void *out[] = {dq, dk, dv, dlog_decay, dstate0};
    const char *names[] = {"dq", "dk", "dv", "dlog_decay", "dstate0"};
    for (int i = 0; i < 5; ++i) {
        if ((rc = check_alias(out[i], names[i], in, 7))) return rc;
        for (int j = 0; j < i; ++j)
            if (out[i] && out[i] == out[j]) { set_error("%s and %s may not be the same memory", names[j], names[i]); return DEER_ERR_INVALID_ARG; }
    }
    if ((rc = check_ws(ws, ws_bytes, carve_lin(nullptr, s, B, T, DEER_OP_ADJOINT).bytes))) return rc;
    const LinWs w = carve_lin(ws, s, B, T, DEER_OP_ADJOINT);
    const int r = s->H / s->Hk, Dk = s->Dk, Dv = s->Dv;
    const bool shared = r > 1, decay = dlog_decay != nullptr;
    const LinView vq = view_of(q, r, T), vk = view_of(k, r, T), vv = view_of(v, 1, T), vg = view_of(g, 1, T);
    LinRole ro[3] = {};
    // dq: the state is S^T [Dv, Dk]
    ro[0].q = vg, ro[0].k = vv, ro[0].v = vk;
    ro[0].Kd = Dv, ro[0].N = Dk;
    ro[0].sc_kv = 1.f, ro[0].sc_o = s->scale;
    ro[0].out = shared ? (void *)w.dq : dq, ro[0].out_f32 = shared, ro[0].wide_out = wide_out(ro[0].out, Dk);
    ro[0].init = state0, ro[0].init_d = 1, ro[0].init_n = Dv;
    if (decay) ro[0].partner = vq, ro[0].dot = w.dq_dot, ro[0].anchor = w.fwd;
    // dk: the state is R^T [Dv, Dk]
    ro[1].q = vv, ro[1].k = vg, ro[1].v = vq;
    ro[1].Kd = Dv, ro[1].N = Dk;
    ro[1].reverse = true;
    ro[1].sc_kv = s->scale, ro[1].sc_o = 1.f;
    ro[1].out = shared ? (void *)w.dk : dk, ro[1].out_f32 = shared, ro[1].wide_out = wide_out(ro[1].out, Dk);
    ro[1].init = g_state, ro[1].init_d = 1, ro[1].init_n = Dv;
    if (decay) ro[1].partner = vk, ro[1].dot = w.dk_dot, ro[1].anchor = w.rev;
    // dv: the state is R [Dk, Dv]
    ro[2].q = vk, ro[2].k = vq, ro[2].v = vg;
    ro[2].Kd = Dk, ro[2].N = Dv;
    ro[2].reverse = true;
    ro[2].sc_kv = s->scale, ro[2].sc_o = 1.f;
    ro[2].out = dv, ro[2].wide_out = wide_out(dv, Dv);
    ro[2].init = g_state, ro[2].init_d = Dv, ro[2].init_n = 1;
    ro[2].fin = dstate0, ro[2].fin_d = Dv, ro[2].fin_n = 1;
    LinArgs a = args_of(s, B, T, DEER_OP_ADJOINT, log_decay, lengths);
    hipStream_t st = (hipStream_t)stream;
    const bool same = lin_same_tile(Dv, Dk, Dk, Dv);
    if (a.nseg > 1) {
        ro[0].seg = w.seg, ro[0].seg_decay = w.seg_decay, ro[0].seg_d = Dk, ro[0].seg_n = 1;
        ro[2].seg = w.rseg, ro[2].seg_decay = w.rseg_decay, ro[2].seg_d = Dv, ro[2].seg_n = 1;
        const LinRole two[2] = {ro[0], ro[2]};
        if (same) {
            if ((rc = launch_lin_walk(a, two, 2, true, false, st))) return rc;
        } else if ((rc = launch_lin_walk(a, two, 1, true, false, st)) ||
                   (rc = launch_lin_walk(a, two + 1, 1, true, false, st))) {
            return rc;
        }
        a.joined = a.nseg > kMostUnjoined;
        if (a.joined && (rc = launch_lin_join(a, two, 2, st))) return rc;
        ro[1].seg = w.rseg, ro[1].seg_decay = w.rseg_decay;
        ro[1].seg_d = 1, ro[1].seg_n = Dv;                       // R^T: the same states, read across
    }
    // Where one tile shape serves all three roles they run in one launch, though dv leaves no dots or
    // anchors (1 x 200 steps, 8 heads of 128 x 128 in bf16: 43 us, dv apart 57; 4 x 4096 steps, 16 heads: 331
    // and 351; in float32, where blocks of dots are slower, 752 and 728, narrower heads 360 and 377).
    if (same) {
        if ((rc = launch_lin_walk(a, ro, 3, false, decay, st))) return rc;
    } else if ((rc = launch_lin_walk(a, ro, 2, false, decay, st)) || (rc = launch_lin_walk(a, ro + 2, 1, false, false, st))) {
        return rc;
    }
    if (shared && (rc = launch_lin_head_sum(s->dtype, (size_t)B * T, s->Hk, r, Dk, w.dq, w.dk, dq, dk, st))) return rc;
    if (!decay) return DEER_OK;
    const int tiles = lin_tiles(Dv, Dk);
    return launch_lin_decay_grad(a, w.dq_dot, tiles, w.dk_dot, tiles, w.fwd, w.rev, Dk * Dv, !state0, w.part, dlog_decay, st);
}

int deer_linattn_step(const deer_linattn_shape *s, int B, const deer_view *q, const deer_view *k, const deer_view *v,
                      const float *log_decay, const int32_t *lengths, float *state, void *o, void *stream) {
    set_error("");
    int rc = check_shape(s, B, 1);
    if (rc) return rc;
    if ((rc = check_view(q, "q", 1)) || (rc = check_view(k, "k", 1)) || (rc = check_view(v, "v", 1))) return rc;
    if (!log_decay || !state || !o) { set_error("log_decay, state and o are required"); return DEER_ERR_INVALID_ARG; }
    const void *in[] = {q->p, k->p, v->p, log_decay};
    if ((rc = check_alias(o, "o", in, 4)) || (rc = check_alias(state, "state", in, 4))) return rc;
    if ((void *)state == o) { set_error("o and state may not be the same memory"); return DEER_ERR_INVALID_ARG; }
    const int r = s->H / s->Hk;
    LinStep a{s->dtype, B, s->H, s->Hk, s->Dk, s->Dv, s->per_step != 0, s->scale, view_of(q, r, 1), view_of(k, r, 1),
              view_of(v, 1, 1), log_decay, lengths, state, o};
    return launch_lin_step(a, (hipStream_t)stream);
}

int deer_layernorm(const deer_norm *n, int64_t rows, const void *x, void *y, float *mean, float *rstd, void *stream) {
    set_error("");
    int rc = check_norm(n, rows);
    if (rc) return rc;
    if (!x || !y) { set_error("x and y are required"); return DEER_ERR_INVALID_ARG; }
    const void *in[] = {x, n->w, n->b};
    if ((rc = check_alias(y, "y", in, 3)) || (rc = check_alias(mean, "mean", in, 3)) ||
        (rc = check_alias(rstd, "rstd", in, 3)))
        return rc;
    if ((mean && mean == rstd) || (void *)mean == y || (void *)rstd == y) {
        set_error("y, mean and rstd may not be the same memory");
        return DEER_ERR_INVALID_ARG;
    }
    return launch_layernorm(norm_of(n, rows, x), y, mean, rstd, (hipStream_t)stream);
}

size_t deer_layernorm_workspace_bytes(const deer_norm *n, int64_t rows) {
    if (check_norm(n, rows) != DEER_OK) return 0;
    return layernorm_adjoint_ws_bytes(norm_of(n, rows, nullptr));
}

int deer_layernorm_adjoint(const deer_norm *n, int64_t rows, const void *x, const void *g, const float *mean,
                           const float *rstd, void *dx, float *dw, float *db, void *ws, size_t ws_bytes, void *stream) {
    set_error("");
    int rc = check_norm(n, rows);
    if (rc) return rc;
    if (!x || !g || !mean || !rstd) { set_error("x, g, mean and rstd are required"); return DEER_ERR_INVALID_ARG; }
    const void *in[] = {x, g, mean, rstd, n->w};
    if ((rc = check_alias(dx, "dx", in, 5)) || (rc = check_alias(dw, "dw", in, 5)) || (rc = check_alias(db, "db", in, 5)))
        return rc;
    if ((dw && dw == db) || (dx && (dx == (void *)dw || dx == (void *)db))) {
        set_error("dx, dw and db may not be the same memory");
        return DEER_ERR_INVALID_ARG;
    }
    if ((rc = check_ws(ws, ws_bytes, layernorm_adjoint_ws_bytes(norm_of(n, rows, x))))) return rc;
    return launch_layernorm_adjoint(norm_of(n, rows, x), g, mean, rstd, dx, dw, db, ws, (hipStream_t)stream);
}

}  // extern "C"
