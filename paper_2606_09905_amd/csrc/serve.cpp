// serve.cpp -- the operators of a language model's layer: 8-bit products with
// token and channel scales, and linear attention with a decay a head.
// Argument checks, planning and the C entry points; the kernels are in
// k_i8s.hip and k_lin.hip.
//
// The one-shot calls keep nothing: each plans its launches (host arithmetic
// only) and enqueues them with the workspace its caller brings, so they may
// be captured, run on any number of streams, and never allocate.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>

#include "plan.h"

using namespace qx;

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 23;
constexpr int64_t kMaxCols = (int64_t)1 << 22;
// |a w| <= 128^2: the int32 sum cannot wrap
constexpr int64_t kMaxK8 = 131071;
constexpr int64_t kMaxHead = 256;
constexpr int64_t kMaxStride = (int64_t)1 << 40;

uint64_t round_up(uint64_t v, uint64_t a) { return (v + a - 1) / a * a; }

// No exception leaves a C entry.
template <class F>
qx_status entry(F&& f) {
    plan_clear_error();
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return plan_fail(QX_ERR_OUT_OF_MEMORY, "host memory");
    } catch (...) {
        return plan_fail(QX_ERR_DEVICE, "unexpected host error");
    }
}

// The type as the caller passed it (any int may stand behind a C enum).
qx_status check_type(const qx_float_type& dt, int32_t* out) {
    static_assert(sizeof(qx_float_type) == sizeof(int32_t), "enum passed as int");
    memcpy(out, &dt, sizeof *out);
    if (*out != FT_F32 && *out != FT_F16 && *out != FT_BF16)
        return plan_fail(QX_ERR_INVALID_ARG, "type %d is not QX_FT_F32, QX_FT_F16 or QX_FT_BF16", *out);
    return QX_OK;
}
uint64_t size_of(int32_t type) { return type == FT_F32 ? 4 : 2; }

qx_status check_size(const char* name, int64_t v, int64_t lo, int64_t hi) {
    if (v < lo) return plan_fail(QX_ERR_INVALID_ARG, "%s = %lld: at least %lld", name, (long long)v, (long long)lo);
    if (v > hi) return plan_fail(QX_ERR_UNSUPPORTED, "%s = %lld exceeds %lld", name, (long long)v, (long long)hi);
    return QX_OK;
}

qx_status check_flag(const char* name, int32_t v) {
    if (v != 0 && v != 1) return plan_fail(QX_ERR_INVALID_ARG, "%s = %d must be 0 or 1", name, v);
    return QX_OK;
}

qx_status check_ws(const Plan& pl, const void* ws, int64_t bytes) {
    const int64_t need = pl.info.workspace_bytes;
    if (need == 0) return QX_OK;
    if (!ws) return plan_fail(QX_ERR_INVALID_ARG, "workspace is NULL; this call needs %lld bytes", (long long)need);
    if (bytes < need)
        return plan_fail(QX_ERR_INVALID_ARG, "workspace of %lld bytes; this call needs %lld", (long long)bytes,
                         (long long)need);
    if ((uintptr_t)ws % 16) return plan_fail(QX_ERR_INVALID_ARG, "workspace is not 16-byte aligned");
    return QX_OK;
}

// A grid holds fewer than 2^32 threads.
qx_status check_grid(int64_t workgroups, int64_t threads) {
    if (workgroups > 0xFFFFFFFFll / threads) return plan_fail(QX_ERR_UNSUPPORTED, "B*H is too large for one launch over heads of these sizes");
    return QX_OK;
}

bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }

// ---------------------------------------------------------------------------
// 8-bit products
// ---------------------------------------------------------------------------
qx_status plan_quant(Plan* pl, int32_t type, int64_t rows, int64_t cols, int64_t ld) {
    qx_status st;
    if ((st = check_size("rows", rows, 0, kMaxRows)) || (st = check_size("cols", cols, 0, kMaxCols))) return st;
    if (ld < cols || ld > kMaxStride)
        return plan_fail(QX_ERR_INVALID_ARG, "ld_x = %lld: at least cols, at most 2^40", (long long)ld);
    pl->op = OP_QUANT_I8;
    pl->n_inputs = 2;
    pl->in_align = size_of(type);
    pl->in_align_of[1] = 4;
    pl->out_align = 1;
    if (rows == 0) return QX_OK;
    QuantI8Params q{};
    q.rows = rows; q.cols = cols; q.ld = ld; q.ldq = cols;
    q.type = type;
    LaunchRec r;
    build_quant_i8(q, &r);
    if (cols) {
        r.bind(offsetof(QuantI8Params, x), BIND_IN0);
        r.bind(offsetof(QuantI8Params, q), BIND_OUT);
    }
    r.bind(offsetof(QuantI8Params, scale), BIND_IN1);
    pl->launches.push_back(r);
    pl->info.tile_m = 1; pl->info.tile_n = (int32_t)std::min<int64_t>(cols, INT32_MAX); pl->info.tile_k = 1;
    pl->info.kernels = 1;
    return QX_OK;
}

qx_status check_product(int64_t M, int64_t N, int64_t K) {
    qx_status st;
    if ((st = check_size("M", M, 0, kMaxRows)) || (st = check_size("N", N, 0, kMaxRows)) ||
        (st = check_size("K", K, 0, kMaxK8)))
        return st;
    if (M && N > ((int64_t)1 << 37) / M) return plan_fail(QX_ERR_UNSUPPORTED, "M*N exceeds 2^37");
    return QX_OK;
}

qx_status plan_gemm_i8s(Plan* pl, int32_t type, int64_t M, int64_t N, int64_t K, bool bias, bool aligned) {
    qx_status st = check_product(M, N, K);
    if (st) return st;
    pl->op = OP_GEMM_I8S;
    pl->n_inputs = 5;
    pl->in_align = 4;
    pl->in_align_of[0] = pl->in_align_of[1] = aligned && K % 16 == 0 ? 16 : 1;
    pl->out_align = size_of(type);
    pl->info.route = R_I8_DIRECT;
    pl->info.products = 1;
    pl->info.exact_no_wrap = 1;
    if (M == 0 || N == 0) return QX_OK;
    GemmI8sParams g{};
    g.lda = std::max<int64_t>(K, 1);
    g.ldw = K;
    g.M = (int32_t)M; g.N = (int32_t)N; g.K = (int32_t)K;
    g.type = type;
    LaunchRec r;
    build_gemm_i8s(g, aligned, &r, &pl->info.tile_m, &pl->info.tile_n, &pl->info.tile_k);
    if (K) {
        r.bind(offsetof(GemmI8sParams, A), BIND_IN0);
        r.bind(offsetof(GemmI8sParams, W), BIND_IN1);
    }
    r.bind(offsetof(GemmI8sParams, sa), BIND_IN2);
    r.bind(offsetof(GemmI8sParams, sw), BIND_IN3);
    if (bias) r.bind(offsetof(GemmI8sParams, bias), BIND_IN4);
    r.bind(offsetof(GemmI8sParams, Y), BIND_OUT);
    pl->launches.push_back(r);
    pl->info.kernels = 1;
    return QX_OK;
}

// Few tokens in one launch; more are quantised into the workspace, then the
// product on them.
qx_status plan_linear_i8(Plan* pl, int32_t type, int64_t M, int64_t N, int64_t K, int64_t ldx, bool bias,
                         bool aligned) {
    qx_status st = check_product(M, N, K);
    if (st) return st;
    if (ldx < K || ldx > kMaxStride)
        return plan_fail(QX_ERR_INVALID_ARG, "ld_x = %lld: at least K, at most 2^40", (long long)ldx);
    pl->op = OP_LINEAR_I8;
    pl->n_inputs = 4;
    pl->in_align = 4;
    pl->in_align_of[0] = (uint8_t)size_of(type);
    pl->in_align_of[1] = aligned && K % 16 == 0 ? 16 : 1;
    pl->out_align = size_of(type);
    pl->info.route = R_I8_DIRECT;
    pl->info.products = 1;
    pl->info.exact_no_wrap = 1;
    if (M == 0 || N == 0) return QX_OK;
    if (fused_i8s(M, K)) {
        GemmI8sParams g{};
        g.ldx = ldx;
        g.ldw = K;
        g.M = (int32_t)M; g.N = (int32_t)N; g.K = (int32_t)K;
        g.type = type;
        LaunchRec r;
        build_gemm_i8s(g, aligned, &r, &pl->info.tile_m, &pl->info.tile_n, &pl->info.tile_k);
        if (K) {
            r.bind(offsetof(GemmI8sParams, x), BIND_IN0);
            r.bind(offsetof(GemmI8sParams, W), BIND_IN1);
        }
        r.bind(offsetof(GemmI8sParams, sw), BIND_IN2);
        if (bias) r.bind(offsetof(GemmI8sParams, bias), BIND_IN3);
        r.bind(offsetof(GemmI8sParams, Y), BIND_OUT);
        pl->launches.push_back(r);
        pl->info.kernels = 1;
        return QX_OK;
    }
    const int64_t ldq = (int64_t)round_up((uint64_t)std::max<int64_t>(K, 1), 16);
    const uint64_t s_off = round_up((uint64_t)M * ldq, 256);
    uint64_t ws = s_off + 4 * (uint64_t)M;
    QuantI8Params q{};
    q.rows = M; q.cols = K; q.ld = ldx; q.ldq = ldq;
    q.type = type;
    // Rows of W that start anywhere cannot go to LDS directly: beyond a few
    // tokens they are copied to whole rows beside the quantisation, but not many
    // rows for few tokens, whose copies take longer than the products gain
    // (copied / not, us: 777 x 1000 x 1501 14.8 / 16.4, 33 x 1000 x 4099 19.9 /
    // 24.8, 256 x 12288 x 8001 86.8 / 94.3, 33 x 16384 x 1001 17.3 / 13.3, 256 x
    // 32768 x 4099 102 / 82, 33 x 32768 x 8001 166 / 79, 512 x 16384 x 4099 77.0
    // / 76.2, 1024 x 16384 x 4099 113 / 117, 2048 x 32768 x 1001 166 / 198)
    const bool copy = K % 16 != 0 && !rows_i8s(M) && (M > 512 || N < 16384);
    uint64_t w_off = 0;
    if (copy) {
        w_off = round_up(ws, 256);
        ws = w_off + (uint64_t)N * ldq;
        q.wrows = N;
    }
    LaunchRec r1, r2;
    build_quant_i8(q, &r1);
    if (K) r1.bind(offsetof(QuantI8Params, x), BIND_IN0);
    r1.bind(offsetof(QuantI8Params, q), BIND_WS, 0);
    r1.bind(offsetof(QuantI8Params, scale), BIND_WS, s_off);
    GemmI8sParams g{};
    g.lda = ldq;
    g.ldw = copy ? ldq : K;
    g.M = (int32_t)M; g.N = (int32_t)N; g.K = (int32_t)K;
    g.type = type;
    build_gemm_i8s(g, copy || aligned, &r2, &pl->info.tile_m, &pl->info.tile_n, &pl->info.tile_k);
    r2.bind(offsetof(GemmI8sParams, A), BIND_WS, 0);
    if (copy) {
        r1.bind(offsetof(QuantI8Params, wsrc), BIND_IN1);
        r1.bind(offsetof(QuantI8Params, wdst), BIND_WS, w_off);
        r2.bind(offsetof(GemmI8sParams, W), BIND_WS, w_off);
    } else if (K) {
        r2.bind(offsetof(GemmI8sParams, W), BIND_IN1);
    }
    r2.bind(offsetof(GemmI8sParams, sa), BIND_WS, s_off);
    r2.bind(offsetof(GemmI8sParams, sw), BIND_IN2);
    if (bias) r2.bind(offsetof(GemmI8sParams, bias), BIND_IN3);
    r2.bind(offsetof(GemmI8sParams, Y), BIND_OUT);
    pl->launches = {r1, r2};
    pl->info.kernels = 2;
    pl->info.workspace_bytes = (int64_t)ws;
    return QX_OK;
}

// ---------------------------------------------------------------------------
// Linear attention
// ---------------------------------------------------------------------------
struct LinSpec {
    int32_t type;
    int64_t B, H, L, dk, dv;
    float scale;
};

qx_status check_lin(const LinSpec& s) {
    qx_status st;
    if ((st = check_size("B", s.B, 0, (int64_t)1 << 24)) || (st = check_size("H", s.H, 0, (int64_t)1 << 24)) ||
        (st = check_size("L", s.L, 0, (int64_t)1 << 30)) || (st = check_size("dk", s.dk, 1, kMaxHead)) ||
        (st = check_size("dv", s.dv, 1, kMaxHead)))
        return st;
    if (s.B * s.H > ((int64_t)1 << 24)) return plan_fail(QX_ERR_UNSUPPORTED, "B*H exceeds 2^24");
    if (!std::isfinite(s.scale)) return plan_fail(QX_ERR_INVALID_ARG, "scale must be finite");
    return QX_OK;
}

// Strides (batch, head[, row]) of one tensor, dense where the caller gives
// none.  Two elements of an output may not share an address.
qx_status take_strides(const char* name, const int64_t* given, const LinSpec& s, int64_t d, bool token, bool out,
                       int64_t* to) {
    const int n = token ? 2 : 3;
    const int64_t rows = token ? 1 : s.L;
    if (!given) {
        to[0] = s.H * rows * d;
        to[1] = rows * d;
        if (!token) to[2] = d;
        return QX_OK;
    }
    const int64_t size[3] = {s.B, s.H, rows};
    for (int i = 0; i < n; ++i) {
        if (given[i] < 0 || given[i] > kMaxStride)
            return plan_fail(QX_ERR_INVALID_ARG, "%s: stride %lld outside [0, 2^40]", name, (long long)given[i]);
        to[i] = given[i];
    }
    if (out) {
        int at[3] = {0, 1, 2};
        std::sort(at, at + n, [&](int a, int b) { return to[a] < to[b]; });
        double extent = (double)d;   // elements that the dimensions so far span
        for (int k = 0; k < n; ++k) {
            const int i = at[k];
            if (size[i] <= 1) continue;
            if ((double)to[i] < extent)
                return plan_fail(QX_ERR_INVALID_ARG, "%s: strides let two of its elements share an address", name);
            extent += (double)to[i] * (double)(size[i] - 1);
        }
    }
    return QX_OK;
}

void note_lin(Plan* pl, const LinShape& sh) {
    pl->info.route = R_LIN_MFMA;
    pl->info.products = 1;
    pl->info.tile_m = 32;
    pl->info.tile_n = 32 * sh.waves;
    pl->info.tile_k = sh.dxp;
    pl->info.k_splits = sh.nseg > 1 ? sh.nseg : 0;
}

// Where one recurrence's operands are bound.
struct LinBinds {
    Bind x, y, z, g;
    int s0, lens, se;   // input index or -1
    Bind o;
    bool in_place;      // se may be the array s0
};

// The launches of one recurrence, appended to the plan.  `states`: the shape
// of the recurrence whose states are this one's, transposed, and lie in the
// workspace already (cut into the same segments).
qx_status add_lin(Plan* pl, const LinSpec& s, LinParams p, const LinBinds& b, const LinShape* states = nullptr) {
    LinShape sh = lin_shape(s.type, p.B, p.H, p.L, p.dx, p.dz);
    if (states) {
        sh.nseg = states->nseg;
        sh.seg_len = states->seg_len;
        sh.u_floats = 0;
        if (sh.nseg > 1) {
            p.u_waves = states->waves;
            p.u_at = states->dxp / 32;
            p.u_nz = states->nz;
        }
    }
    const qx_status st = check_grid((int64_t)p.B * p.H * sh.nz * sh.nseg, 64 * sh.waves);
    if (st) return st;
    if (sh.u_floats) {
        const qx_status st2 = check_grid(sh.u_floats / 4 / sh.nseg / 256, 256);
        if (st2) return st2;
    }
    // Without a scan every segment reads S0 and the states before it: at most
    // eight segments, and 16 MiB in all (64 KiB a state of 128 x 128); not where
    // the last segment may meanwhile write its end over S0 (16 heads x 512 x
    // 64 fp16: 30 -> 24 us)
    p.prefix = !states && !b.in_place && sh.nseg > 1 && sh.nseg <= 8 && sh.u_floats * sh.nseg <= (int64_t)8 << 20;
    auto bind = [&](LaunchRec& r, bool scan, bool out) {
        if (!scan && s.L) {
            if (out) r.bind(offsetof(LinParams, X), b.x);
            r.bind(offsetof(LinParams, Y), b.y);
            r.bind(offsetof(LinParams, Z), b.z);
            if (out) r.bind(offsetof(LinParams, O), b.o);
        }
        r.bind(offsetof(LinParams, g), b.g);
        if (b.lens >= 0) r.bind(offsetof(LinParams, lens), (Bind)b.lens);
        if (b.s0 >= 0 && (scan || (out && (sh.nseg == 1 || p.prefix)))) r.bind(offsetof(LinParams, S0), (Bind)b.s0);
        if (b.se >= 0 && out) r.bind(offsetof(LinParams, SE), (Bind)b.se);
        if (sh.nseg > 1) r.bind(offsetof(LinParams, U), BIND_WS, 0);
    };
    if (sh.nseg > 1 && !states) {
        LaunchRec r1, r2;
        build_lin(s.type, sh, p, true, &r1);
        bind(r1, false, false);
        pl->launches.push_back(r1);
        if (!p.prefix) {
            build_lin_scan(sh, p, &r2);
            bind(r2, true, false);
            pl->launches.push_back(r2);
        }
    }
    LaunchRec r;
    build_lin(s.type, sh, p, false, &r);
    bind(r, false, true);
    pl->launches.push_back(r);
    pl->info.kernels = (int32_t)pl->launches.size();
    pl->info.workspace_bytes = std::max(pl->info.workspace_bytes, (int64_t)(4 * sh.u_floats));
    note_lin(pl, sh);
    return QX_OK;
}

// inputs {Q, K, V, log_decay, S0, lens, S_out}, output O (S_out where L is 0)
qx_status plan_lin_attn(Plan* pl, const LinSpec& s, const int64_t* strides, bool state, bool lens, bool end,
                        bool in_place) {
    qx_status st = check_lin(s);
    if (st) return st;
    LinParams p{};
    if ((st = take_strides("Q", strides, s, s.dk, false, false, p.sx)) ||
        (st = take_strides("K", strides ? strides + 3 : nullptr, s, s.dk, false, false, p.sy)) ||
        (st = take_strides("V", strides ? strides + 6 : nullptr, s, s.dv, false, false, p.sz)) ||
        (st = take_strides("O", strides ? strides + 9 : nullptr, s, s.dv, false, true, p.so)))
        return st;
    const uint8_t es = (uint8_t)size_of(s.type);
    pl->op = OP_LIN_ATTN;
    pl->n_inputs = 7;
    pl->in_align = 4;
    for (int i : {0, 1, 2}) pl->in_align_of[i] = es;
    pl->out_align = es;
    pl->info.route = R_LIN_MFMA;
    if (s.B == 0 || s.H == 0 || (s.L == 0 && !end)) return QX_OK;
    p.B = (int32_t)s.B; p.H = (int32_t)s.H; p.L = (int32_t)s.L;
    p.dx = (int32_t)s.dk; p.dz = (int32_t)s.dv;
    p.p_mul = p.q_mul = s.scale;
    p.u_mul = 1.f;
    return add_lin(pl, s, p, LinBinds{BIND_IN0, BIND_IN1, BIND_IN2, BIND_IN3, state ? 4 : -1, lens ? 5 : -1, end ? 6 : -1,
                                      BIND_OUT, in_place});
}

// inputs {Q, K, V, dO, log_decay, S0, dS, lens, dQ, dK, dS0}, output dV.
// With G_{n-1} = scale q_{n-1}^T dO_{n-1} + dS, G_i = scale q_i^T dO_i + lambda G_{i+1},
// dS0 = lambda G_0 (dS where there is no token):
//   dQ_i = scale dO_i S_i^T        the forward recurrence on (dO, V, K), S0^T
//   dK_i = V_i G_i^T, dV_i = K_i G_i   backwards on (V, dO, Q), dS^T and (K, Q, dO), dS
qx_status plan_lin_backward(Plan* pl, const LinSpec& s, const int64_t* strides, bool state, bool d_end, bool lens,
                            bool d_state) {
    qx_status st = check_lin(s);
    if (st) return st;
    const char* names[7] = {"Q", "K", "V", "dO", "dQ", "dK", "dV"};
    int64_t sd[7][3];
    for (int i = 0; i < 7; ++i) {
        const int64_t d = i == 2 || i == 3 || i == 6 ? s.dv : s.dk;
        if ((st = take_strides(names[i], strides ? strides + 3 * i : nullptr, s, d, false, i >= 4, sd[i]))) return st;
    }
    const uint8_t es = (uint8_t)size_of(s.type);
    pl->op = OP_LIN_BWD;
    pl->n_inputs = 11;
    pl->in_align = 4;
    for (int i : {0, 1, 2, 3, 8, 9}) pl->in_align_of[i] = es;
    pl->out_align = es;
    pl->info.route = R_LIN_MFMA;
    if (s.B == 0 || s.H == 0 || (s.L == 0 && !d_state)) return QX_OK;
    auto params = [&](int x, int y, int z, int o) {
        LinParams p{};
        const int64_t d[7] = {s.dk, s.dk, s.dv, s.dv, s.dk, s.dk, s.dv};
        std::copy(sd[x], sd[x] + 3, p.sx);
        std::copy(sd[y], sd[y] + 3, p.sy);
        std::copy(sd[z], sd[z] + 3, p.sz);
        std::copy(sd[o], sd[o] + 3, p.so);
        p.B = (int32_t)s.B; p.H = (int32_t)s.H; p.L = (int32_t)s.L;
        p.dx = (int32_t)d[x]; p.dz = (int32_t)d[z];
        p.p_mul = s.scale;
        p.q_mul = p.u_mul = 1.f;
        return p;
    };
    const int ln = lens ? 7 : -1;
    LinParams v = params(1, 0, 3, 6);
    v.u_mul = s.scale;
    v.rev = 1;
    const LinShape shape = lin_shape(s.type, v.B, v.H, v.L, v.dx, v.dz);
    LinParams k = params(2, 3, 0, 5);
    k.u_mul = s.scale;
    k.rev = k.s_t = 1;
    if (s.L) {
        LinParams q = params(3, 2, 1, 4);
        q.q_mul = s.scale;
        q.s_t = 1;
        if ((st = add_lin(pl, s, q, LinBinds{BIND_IN3, BIND_IN2, BIND_IN1, BIND_IN4, state ? 5 : -1, ln, -1, BIND_IN8, false}))) return st;
        // with one segment dK reads dS itself: ahead of dV, which may write dS0 over it
        if (shape.nseg == 1 &&
            (st = add_lin(pl, s, k, LinBinds{BIND_IN2, BIND_IN3, BIND_IN0, BIND_IN4, d_end ? 6 : -1, ln, -1, BIND_IN9, true}, &shape)))
            return st;
    }
    if ((st = add_lin(pl, s, v, LinBinds{BIND_IN1, BIND_IN0, BIND_IN3, BIND_IN4, d_end ? 6 : -1, ln, d_state ? 10 : -1, BIND_OUT, true})))
        return st;
    // G_i at the segments' ends is one thing for dK and dV
    if (shape.nseg > 1)
        return add_lin(pl, s, k, LinBinds{BIND_IN2, BIND_IN3, BIND_IN0, BIND_IN4, -1, ln, -1, BIND_IN9, true}, &shape);
    return QX_OK;
}

// inputs {q, k, v, log_decay, S}, output o
qx_status plan_lin_step(Plan* pl, const LinSpec& s, const int64_t* strides) {
    qx_status st = check_lin(s);
    if (st) return st;
    LinStepParams p{};
    if ((st = take_strides("q", strides, s, s.dk, true, false, p.sq)) ||
        (st = take_strides("k", strides ? strides + 2 : nullptr, s, s.dk, true, false, p.sk)) ||
        (st = take_strides("v", strides ? strides + 4 : nullptr, s, s.dv, true, false, p.sv)) ||
        (st = take_strides("o", strides ? strides + 6 : nullptr, s, s.dv, true, true, p.so)))
        return st;
    const uint8_t es = (uint8_t)size_of(s.type);
    pl->op = OP_LIN_STEP;
    pl->n_inputs = 5;
    pl->in_align = 4;
    for (int i : {0, 1, 2}) pl->in_align_of[i] = es;
    pl->out_align = es;
    pl->info.route = R_LIN_STEP;
    pl->info.products = 1;
    if (s.B == 0 || s.H == 0) return QX_OK;
    p.B = (int32_t)s.B; p.H = (int32_t)s.H;
    p.dk = (int32_t)s.dk; p.dv = (int32_t)s.dv;
    p.scale = s.scale;
    p.type = s.type;
    if ((st = check_grid(s.B * s.H * ((s.dv + 31) / 32), 256))) return st;
    LaunchRec r;
    build_lin_step(p, &r);
    r.bind(offsetof(LinStepParams, q), BIND_IN0);
    r.bind(offsetof(LinStepParams, k), BIND_IN1);
    r.bind(offsetof(LinStepParams, v), BIND_IN2);
    r.bind(offsetof(LinStepParams, g), BIND_IN3);
    r.bind(offsetof(LinStepParams, S), BIND_IN4);
    r.bind(offsetof(LinStepParams, o), BIND_OUT);
    pl->launches.push_back(r);
    pl->info.tile_m = 1; pl->info.tile_n = (int32_t)std::min<int64_t>(s.dv, 128); pl->info.tile_k = (int32_t)s.dk;
    pl->info.kernels = 1;
    return QX_OK;
}

template <class MakePlan>
qx_status query(qx_plan_info* out, MakePlan make) {
    return entry([&] {
        if (!out) return plan_fail(QX_ERR_INVALID_ARG, "out is NULL");
        Plan pl;
        const qx_status st = make(&pl);
        if (!st) *out = pl.info;
        return st;
    });
}

template <class MakePlan>
qx_status create(qx_exec* out, MakePlan make) {
    return entry([&] {
        if (!out) return plan_fail(QX_ERR_INVALID_ARG, "out is NULL");
        *out = nullptr;
        Plan pl;
        const qx_status st = make(&pl);
        return st ? st : plan_create(std::move(pl), out);
    });
}

}  // namespace

// ---------------------------------------------------------------------------
// C ABI
// ---------------------------------------------------------------------------
extern "C" {

qx_status quantize_rows_i8(qx_float_type dt, const void* x, int8_t* q, float* scale, int64_t rows, int64_t cols,
                           int64_t ld_x, void* stream) {
    return entry([&] {
        int32_t t;
        Plan pl;
        qx_status st = check_type(dt, &t);
        if (st || (st = plan_quant(&pl, t, rows, cols, ld_x))) return st;
        const void* in[2] = {x, scale};
        // rows without columns have a scale each and nothing else
        return plan_run(pl, in, cols ? (void*)q : (void*)scale, nullptr, stream);
    });
}

qx_status qgemm_i8_scaled(qx_float_type dt, const int8_t* A, const int8_t* W, const float* scale_a,
                          const float* scale_w, const float* bias, void* Y, int64_t M, int64_t N, int64_t K,
                          void* stream) {
    return entry([&] {
        int32_t t;
        Plan pl;
        qx_status st = check_type(dt, &t);
        if (st || (st = plan_gemm_i8s(&pl, t, M, N, K, bias != nullptr, aligned16(A) && aligned16(W)))) return st;
        const void* in[5] = {A, W, scale_a, scale_w, bias};
        return plan_run(pl, in, Y, nullptr, stream);
    });
}

qx_status linear_i8(qx_float_type dt, const void* x, const int8_t* W, const float* scale_w, const float* bias,
                    void* Y, int64_t M, int64_t N, int64_t K, int64_t ld_x, void* workspace, int64_t workspace_bytes,
                    void* stream) {
    return entry([&] {
        int32_t t;
        Plan pl;
        qx_status st = check_type(dt, &t);
        if (st || (st = plan_linear_i8(&pl, t, M, N, K, ld_x, bias != nullptr, aligned16(W)))) return st;
        if ((st = check_ws(pl, workspace, workspace_bytes))) return st;
        const void* in[4] = {x, W, scale_w, bias};
        return plan_run(pl, in, Y, workspace, stream);
    });
}

qx_status lin_attn(qx_float_type dt, const void* Q, const void* K, const void* V, const float* log_decay,
                   const float* S0, const int32_t* lens, void* O, float* S_out, int64_t B, int64_t H, int64_t L,
                   int64_t dk, int64_t dv, const int64_t* strides, float scale, void* workspace,
                   int64_t workspace_bytes, void* stream) {
    return entry([&] {
        LinSpec s{0, B, H, L, dk, dv, scale};
        Plan pl;
        qx_status st = check_type(dt, &s.type);
        if (st || (st = plan_lin_attn(&pl, s, strides, S0 != nullptr, lens != nullptr, S_out != nullptr,
                                                 S0 != nullptr && S0 == S_out))) return st;
        if ((st = check_ws(pl, workspace, workspace_bytes))) return st;
        const void* in[7] = {Q, K, V, log_decay, S0, lens, S_out};
        return plan_run(pl, in, L ? O : (void*)S_out, workspace, stream);
    });
}

qx_status lin_attn_step(qx_float_type dt, const void* q, const void* k, const void* v, const float* log_decay,
                        float* S, void* o, int64_t B, int64_t H, int64_t dk, int64_t dv, const int64_t* strides,
                        float scale, void* stream) {
    return entry([&] {
        LinSpec s{0, B, H, 1, dk, dv, scale};
        Plan pl;
        qx_status st = check_type(dt, &s.type);
        if (st || (st = plan_lin_step(&pl, s, strides))) return st;
        const void* in[5] = {q, k, v, log_decay, S};
        return plan_run(pl, in, o, nullptr, stream);
    });
}

qx_status lin_attn_backward(qx_float_type dt, const void* Q, const void* K, const void* V, const void* dO,
                            const float* log_decay, const float* S0, const float* dS_out, const int32_t* lens,
                            void* dQ, void* dK, void* dV, float* dS0, int64_t B, int64_t H, int64_t L, int64_t dk,
                            int64_t dv, const int64_t* strides, float scale, void* workspace, int64_t workspace_bytes,
                            void* stream) {
    return entry([&] {
        LinSpec s{0, B, H, L, dk, dv, scale};
        Plan pl;
        qx_status st = check_type(dt, &s.type);
        if (st || (st = plan_lin_backward(&pl, s, strides, S0 != nullptr, dS_out != nullptr, lens != nullptr, dS0 != nullptr)))
            return st;
        if ((st = check_ws(pl, workspace, workspace_bytes))) return st;
        const void* in[11] = {Q, K, V, dO, log_decay, S0, dS_out, lens, dQ, dK, dS0};
        return plan_run(pl, in, L ? dV : (void*)dS0, workspace, stream);
    });
}

// ---- planner queries ------------------------------------------------------

qx_status qx_plan_quantize_rows_i8(qx_plan_info* out, qx_float_type dt, int64_t rows, int64_t cols) {
    return query(out, [&](Plan* pl) {
        int32_t t;
        const qx_status st = check_type(dt, &t);
        return st ? st : plan_quant(pl, t, rows, cols, cols);
    });
}

qx_status qx_plan_gemm_i8_scaled(qx_plan_info* out, qx_float_type dt, int64_t M, int64_t N, int64_t K) {
    return query(out, [&](Plan* pl) {
        int32_t t;
        const qx_status st = check_type(dt, &t);
        return st ? st : plan_gemm_i8s(pl, t, M, N, K, false, true);
    });
}

qx_status qx_plan_linear_i8(qx_plan_info* out, qx_float_type dt, int64_t M, int64_t N, int64_t K) {
    return query(out, [&](Plan* pl) {
        int32_t t;
        const qx_status st = check_type(dt, &t);
        return st ? st : plan_linear_i8(pl, t, M, N, K, K, false, true);
    });
}

qx_status qx_plan_lin_attn(qx_plan_info* out, qx_float_type dt, int64_t B, int64_t H, int64_t L, int64_t dk,
                           int64_t dv) {
    return query(out, [&](Plan* pl) {
        LinSpec s{0, B, H, L, dk, dv, 1.f};
        const qx_status st = check_type(dt, &s.type);
        return st ? st : plan_lin_attn(pl, s, nullptr, true, true, true, true);
    });
}

qx_status qx_plan_lin_attn_step(qx_plan_info* out, qx_float_type dt, int64_t B, int64_t H, int64_t dk, int64_t dv) {
    return query(out, [&](Plan* pl) {
        LinSpec s{0, B, H, 1, dk, dv, 1.f};
        const qx_status st = check_type(dt, &s.type);
        return st ? st : plan_lin_step(pl, s, nullptr);
    });
}

qx_status qx_plan_lin_attn_backward(qx_plan_info* out, qx_float_type dt, int64_t B, int64_t H, int64_t L, int64_t dk,
                                    int64_t dv) {
    return query(out, [&](Plan* pl) {
        LinSpec s{0, B, H, L, dk, dv, 1.f};
        const qx_status st = check_type(dt, &s.type);
        return st ? st : plan_lin_backward(pl, s, nullptr, true, true, true, true);
    });
}

// ---- executors ------------------------------------------------------------

qx_status qx_exec_create_gemm_i8_scaled(qx_exec* out, qx_float_type dt, int64_t M, int64_t N, int64_t K,
                                        int32_t has_bias) {
    return create(out, [&](Plan* pl) {
        int32_t t;
        qx_status st = check_type(dt, &t);
        if (st || (st = check_flag("has_bias", has_bias))) return st;
        st = plan_gemm_i8s(pl, t, M, N, K, has_bias != 0, true);
        pl->n_inputs = has_bias ? 5 : 4;
        return st;
    });
}

qx_status qx_exec_create_linear_i8(qx_exec* out, qx_float_type dt, int64_t M, int64_t N, int64_t K, int32_t has_bias) {
    return create(out, [&](Plan* pl) {
        int32_t t;
        qx_status st = check_type(dt, &t);
        if (st || (st = check_flag("has_bias", has_bias))) return st;
        st = plan_linear_i8(pl, t, M, N, K, K, has_bias != 0, true);
        pl->n_inputs = has_bias ? 4 : 3;
        return st;
    });
}

qx_status qx_exec_create_lin_attn(qx_exec* out, qx_float_type dt, int64_t B, int64_t H, int64_t L, int64_t dk,
                                  int64_t dv, float scale) {
    return create(out, [&](Plan* pl) {
        LinSpec s{0, B, H, L, dk, dv, scale};
        qx_status st = check_type(dt, &s.type);
        // {Q, K, V, log_decay, S}: the state is taken and left in S
        if (st || (st = check_size("L", L, 1, (int64_t)1 << 30)) || (st = plan_lin_attn(pl, s, nullptr, true, false, true, true)))
            return st;
        for (LaunchRec& r : pl->launches)
            for (int i = 0; i < r.nslots; ++i)
                if (r.slots[i].bind == BIND_IN6) r.slots[i].bind = BIND_IN4;
        pl->n_inputs = 5;
        return st;
    });
}

qx_status qx_exec_create_lin_attn_step(qx_exec* out, qx_float_type dt, int64_t B, int64_t H, int64_t dk, int64_t dv,
                                       float scale) {
    return create(out, [&](Plan* pl) {
        LinSpec s{0, B, H, 1, dk, dv, scale};
        const qx_status st = check_type(dt, &s.type);
        return st ? st : plan_lin_step(pl, s, nullptr);
    });
}

}  // extern "C"
