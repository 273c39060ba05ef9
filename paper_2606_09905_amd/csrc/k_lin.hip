// k_lin.hip -- linear attention with a decay for each head.
//
//   S_t = lambda S_{t-1} + y_t^T z_t,   o_t = x_t S_t
//
// over chunks of 32 tokens (prompts, and every part of the backward pass) and
// for one token (serving).
//
// A chunk that starts with state S gives
//   o_i = lambda^{i+1} x_i S + sum_{j<=i} lambda^{i-j} (x_i . y_j) z_j
//   S'  = lambda^32 S + sum_j lambda^{31-j} y_j^T z_j
// which only has powers with exponents >= 0, so any decay, 0 included, is safe.
//
// A wave owns 32 columns of z and walks the chunks on its own: the state
// (dx x 32) stays in its accumulators, and all four products run transposed,
// so that what one leaves in its accumulators is the next one's operand
// without a lane moving:
//   P^T = Y X^T         lane = token i, registers = tokens j
//   O^T = S^T X^T       lane = token i, registers = columns; S^T is the
//                       accumulators of S read as an A operand
//   O^T += Z^T P^T      P^T read as a B operand
//   S  += Y^T (w Z)     Z^T's fragment, scaled, read as a B operand
// The matrix core's own order of the contracted index (4 of every 8) is given
// to both operands.  Y^T and Z^T come from row-major tiles through the
// transposing LDS read.  Every wave of a workgroup forms P itself, 8 of its 52
// products at dx 128, which takes P out of LDS and a barrier out of the chunk.
//
// Precision: operands are exact sums of bf16 terms (bf16 one, fp16 two, fp32
// three).  What is computed on the way (scores, the state as an operand) is
// split into as many terms as the result's type needs, two for the 16-bit
// types (2^-17 of a value), three for fp32; the products that update the
// state, which is fp32 in every type, take three (the whole 24 bits).  Of the
// products of two such sums those are kept whose terms' ranks add up to less
// than the number of terms.
//
// Long sequences of few heads are cut into segments: a first launch forms each
// segment's own state, a scan turns these into the states before the segments,
// and the launch over all chunks starts each segment from its own.
//
// What bounds it: bf16 the memory, of which the segments' states ask for Y and
// Z a second time (64 heads x 8192 x 128: states 66 us for 268 MB, chunks 160
// us for 537 MB, 3.4 TB/s; three streams read and one written in the same
// tiles without any work take 140 us); fp32 the matrix cores and the splitting
// of values into terms, six products for one (64 heads x 1999 x 96 x 80: 115 us),
// and registers in scratch (42 a lane there; 14 at dx 64 with two waves).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "qx_internal.h"

namespace qx {

namespace {

typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16x __attribute__((ext_vector_type(16)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
// vectors at any address: rows may start anywhere
typedef u4 u4u __attribute__((aligned(2)));
typedef u2 u2u __attribute__((aligned(2)));
typedef f4 f4u __attribute__((aligned(4)));

struct Half { uint16_t v; };
struct Bf16 { uint16_t v; };

constexpr int CH = 32;   // tokens of a chunk: one 32 x 32 tile of scores

template <class E> constexpr int kTerms = 1;                // bf16 terms of an operand
template <> constexpr int kTerms<Half> = 2;
template <> constexpr int kTerms<float> = 3;
template <class E> constexpr int kOutTerms = 2;             // of a computed value behind an output
template <> constexpr int kOutTerms<float> = 3;
constexpr int kStateTerms = 3;                              // of a computed value behind the state

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, b2));
}
__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }

// two floats -> N words of two bf16 terms each, every term the rounding of
// what the ones before it leave.  (The remainder as one dot product, which
// takes a term out of its word and subtracts it, measured no better: the
// two-operand form overwrites the float and needs wait states around it.)
template <int N>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t (&w)[N]) {
#pragma unroll
    for (int t = 0; t < N; ++t) {
        w[t] = bf16_pair(a, b);
        if (t + 1 < N) {
            a -= lo_f(w[t]);
            b -= hi_f(w[t]);
        }
    }
}

template <int N>
__device__ __forceinline__ void split8(const float (&x)[8], b8 (&t)[N]) {
    uint32_t w[N][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t v[N];
        split_pair<N>(x[2 * i], x[2 * i + 1], v);
#pragma unroll
        for (int n = 0; n < N; ++n) w[n][i] = v[n];
    }
#pragma unroll
    for (int n = 0; n < N; ++n) t[n] = __builtin_bit_cast(b8, w[n]);
}

// exp(g n), n >= 0: 1 for n = 0 whatever g is (g may be -inf: decay 0)
__device__ __forceinline__ float decay_pow(float g, int n) {
    return n == 0 ? 1.f : __builtin_amdgcn_exp2f((float)((double)g * 1.4426950408889634 * n));
}

// The rounding of a factor close to one is a change of the decay, the same one
// each time it is applied: at g = -1e-6, token by token, 1.3% of it.
//
// One token's: s exp(g) + more, as s + (s (exp(g) - 1) + more) where exp(g) is
// more than a half.
struct Decay {
    float f;      // exp(g) - 1, or exp(g)
    bool near;    // (the same for all threads of a head)
    __device__ __forceinline__ float of(float s, float more) const {
        const float t = __builtin_fmaf(s, f, more);
        return near ? s + t : t;
    }
};
__device__ __forceinline__ Decay decay_of(float g) {
    const bool near = g > -0.69f;
    const float less = expm1f(g), whole = decay_pow(g, 1);   // (both: a branch would hold back the loads behind it)
    return {near ? less : whole, near};
}
// The factors exp(g n) for one step of n tokens after the other: of the two
// floats around it now one, now the other, so that the product of any number
// of them is a rounding off.  (The two terms above for each element of the
// state cost up to 37% of the time of all chunks; of these a wave has two scalar adds.)
struct Factors {
    uint32_t lo, part, at;   // the smaller float; how far, in 2^-32, exp(g n) lies past it; what has gathered
    __device__ __forceinline__ float next() {
        const uint32_t was = at;
        at += part;
        return __uint_as_float(lo + (at < was ? 1u : 0u));
    }
};
__device__ __forceinline__ Factors factors_of(float g, int n) {
    const double x = (double)g * n;
    const bool near = fabs(x) < 0.69;
    const float e = near ? expm1f((float)x) : 0.f;
    const float k = e * (e < 0.f ? 0x1p24f : 0x1p23f), f = floorf(k);   // in places of the floats below or above one
    const uint32_t lo = __float_as_uint(near ? 1.f + f * (e < 0.f ? 0x1p-24f : 0x1p-23f) : decay_pow(g, n));
    const uint32_t part = (uint32_t)fminf((k - f) * 0x1p32f, 4294967040.f);
    return {lo, part, 0x80000000u};
}
__device__ __forceinline__ Factors for_wave(const Factors& f) {
    return {(uint32_t)__builtin_amdgcn_readfirstlane((int)f.lo), (uint32_t)__builtin_amdgcn_readfirstlane((int)f.part), 0x80000000u};
}

// Eight elements: all of them, or the first n with zeros behind them; raw
// 16-bit words or floats.
template <class E>
struct Vec8 {
    uint32_t w[4];
    __device__ __forceinline__ void zero() { w[0] = w[1] = w[2] = w[3] = 0; }
    __device__ __forceinline__ void load8(const void* at) {
        const u4 v = *(const u4u*)at;
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    }
    __device__ __forceinline__ void load(const void* at, int n) {
        if (n >= 8) {
            load8(at);
        } else {
            const uint16_t* q = (const uint16_t*)at;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = (2 * i < n ? q[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)q[2 * i + 1] : 0u) << 16;
        }
    }
};
template <>
struct Vec8<float> {
    float w[8];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 0.f;
    }
    __device__ __forceinline__ void load8(const void* at) {
        const f4 a = *(const f4u*)at, b = *(const f4u*)((const float*)at + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { w[i] = a[i]; w[4 + i] = b[i]; }
    }
    __device__ __forceinline__ void load(const void* at, int n) {
        if (n >= 8) {
            load8(at);
        } else {
            const float* q = (const float*)at;
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = i < n ? q[i] : 0.f;
        }
    }
};

// A vector's terms, and whether all of it is finite: an infinity or NaN keeps
// only its first term, since the others would be NaN.  (By selections: a branch
// around the mending of such vectors measured 12% slower, fp32 at dx 96.)
__device__ __forceinline__ bool terms_of(const Vec8<Bf16>& v, u4 (&t)[1]) {
    t[0] = u4{v.w[0], v.w[1], v.w[2], v.w[3]};
    // the largest magnitudes of both halves: 16-bit integers order like them
    typedef uint16_t us2 __attribute__((ext_vector_type(2)));
    us2 m = __builtin_bit_cast(us2, v.w[0] & 0x7FFF7FFFu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(us2, v.w[i] & 0x7FFF7FFFu));
    return max(m.x, m.y) < 0x7F80;
}
template <int N>
__device__ __forceinline__ bool float_terms(const float (&x)[8], u4 (&t)[N]) {
    bool ok = true;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = x[2 * i], b = x[2 * i + 1];
        const uint32_t h = bf16_pair(a, b);
        const bool fa = finite(lo_f(h)), fb = finite(hi_f(h));
        ok = ok && fa && fb;
        t[0][i] = h;
#pragma unroll
        for (int n = 1; n < N; ++n) {
            a -= lo_f(t[n - 1][i]);
            b -= hi_f(t[n - 1][i]);
            t[n][i] = bf16_pair(fa ? a : 0.f, fb ? b : 0.f);
        }
    }
    return ok;
}
__device__ __forceinline__ bool terms_of(const Vec8<Half>& v, u4 (&t)[2]) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)v.w[i]);
        x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(v.w[i] >> 16));
    }
    return float_terms<2>(x, t);
}
__device__ __forceinline__ bool terms_of(const Vec8<float>& v, u4 (&t)[3]) { return float_terms<3>(v.w, t); }

// four consecutive outputs of a row, as words of the result's type
template <class E> struct Out4 { uint32_t w[2]; };
template <> struct Out4<float> { uint32_t w[4]; };
__device__ __forceinline__ Out4<Bf16> round4(Bf16*, const float (&x)[4]) {
    return {{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])}};
}
__device__ __forceinline__ Out4<Half> round4(Half*, const float (&x)[4]) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    return {{__builtin_bit_cast(uint32_t, h2{(_Float16)x[0], (_Float16)x[1]}),
             __builtin_bit_cast(uint32_t, h2{(_Float16)x[2], (_Float16)x[3]})}};
}
__device__ __forceinline__ Out4<float> round4(float*, const float (&x)[4]) {
    return {{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])}};
}
template <class E>
__device__ __forceinline__ void store4(void* row, int c, int d, const Out4<E>& v) {
    if constexpr (sizeof(E) == 4) {
        uint32_t* q = (uint32_t*)row + c;
        if (c + 4 <= d) {
            *(u4u*)q = u4{v.w[0], v.w[1], v.w[2], v.w[3]};
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (c + i < d) q[i] = v.w[i];
        }
    } else {
        uint16_t* q = (uint16_t*)row + c;
        if (c + 4 <= d) {
            *(u2u*)q = u2{v.w[0], v.w[1]};
        } else {
            if (c < d) q[0] = (uint16_t)v.w[0];
            if (c + 1 < d) q[1] = (uint16_t)(v.w[0] >> 16);
            if (c + 2 < d) q[2] = (uint16_t)v.w[1];
        }
    }
}

__device__ __forceinline__ s4 read_tr(const uint16_t* a) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)a);
}
__device__ __forceinline__ b8 join(s4 a, s4 b) {
    const u2 x = __builtin_bit_cast(u2, a), y = __builtin_bit_cast(u2, b);
    return __builtin_bit_cast(b8, u4{x.x, x.y, y.x, y.y});
}

__device__ __forceinline__ f16x mfma(b8 a, b8 b, f16x c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// acc += sum of the products of a's and b's terms whose ranks add up to less
// than MAXT
template <int NA, int NB, int MAXT>
__device__ __forceinline__ void mma(f16x& acc, const b8 (&a)[NA], const b8 (&b)[NB]) {
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
            if (i + j < MAXT) acc = mfma(a[i], b[j], acc);
}
// two such sums in turn: a product waits for the one before it in its own sum
template <int NA, int NB, int MAXA, int NC, int ND, int MAXC>
__device__ __forceinline__ void mma2(f16x& acc, const b8 (&a)[NA], const b8 (&b)[NB], f16x& acc2, const b8 (&c)[NC],
                                     const b8 (&d)[ND]) {
    constexpr int N = NA * NB > NC * ND ? NA * NB : NC * ND;
#pragma unroll
    for (int q = 0; q < N; ++q) {
        if (q < NC * ND && q / ND + q % ND < MAXC) acc2 = mfma(c[q / ND], d[q % ND], acc2);
        if (q < NA * NB && q / NB + q % NB < MAXA) acc = mfma(a[q / NB], b[q % NB], acc);
    }
}

}  // namespace

// The chunks of one segment of one head, for 32 W columns of z.
// STATE: only the segment's own state, into U.
// VEC: rows are whole vectors of eight elements.
template <class E, int DX, int W, bool STATE, bool VEC>
__global__ __launch_bounds__(64 * W, DX <= 128 ? 2 : 1) void k_lin(const LinParams p) {
    constexpr int T = kTerms<E>, NS = kOutTerms<E>, MS = NS > T ? NS : T;
    // Rows of X and Y are 56, 184 or 200 bytes past a multiple of 256 apart: 32
    // rows then start in 32 different pairs of the 64 banks (their reads by
    // row), and any four lie next to each other (the transposing reads of 64
    // bytes from each of four rows).  Z's only has the latter.
    constexpr int NTH = 64 * W, ZW = 32 * W, AT = DX / 32;
    constexpr int DXP = DX + (DX == 96 ? 4 : 28), ZP = ZW + 32;
    constexpr int VX = CH * DX / 8, VZ = CH * ZW / 8;      // vectors of a tile
    constexpr int NX = (VX + NTH - 1) / NTH, NZ = VZ / NTH;
    constexpr int64_t ES = sizeof(E);
    static_assert(VZ % NTH == 0, "whole z tile");
    // the next chunk's rows are held in registers while this one is computed
    // where they are few, and go to a second buffer where LDS holds two
    // workgroups' pairs of them: one barrier a chunk instead of two
    constexpr bool AHEAD = (STATE ? NX + NZ : 2 * NX + NZ) * (int)sizeof(Vec8<E>) / 4 <= 64;
    constexpr int TILE = T * CH * ((STATE ? 1 : 2) * DXP + ZP) * 2;
    constexpr int NB = AHEAD && 2 * TILE <= 78 * 1024 ? 2 : 1;
    __shared__ __align__(16) uint16_t Xs[NB][STATE ? 1 : T][STATE ? 1 : CH][STATE ? 8 : DXP];
    __shared__ __align__(16) uint16_t Ys[NB][T][CH][DXP];
    __shared__ __align__(16) uint16_t Zs[NB][T][CH][ZP];
    __shared__ float pw[CH + 1], pu[2 * CH];               // powers of the decay; the update's weights
    __shared__ Factors fs;                                 // of a whole chunk
    __shared__ int odd[2];                                 // the last chunk (of even and odd ones) whose z is not finite

    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int id = blockIdx.x;
    const int seg = id % p.nseg;
    id /= p.nseg;
    const int zt = id % p.nz, bh = id / p.nz;
    const int b = bh / p.H, h = bh - b * p.H;
    const int len = p.lens ? min(max(p.lens[b], 0), p.L) : p.L;
    const int t0 = seg * p.seg_len;
    // a segment's own state is asked for by the segments behind it only
    if (STATE ? t0 + p.seg_len >= len : seg > 0 && t0 >= len) return;
    const int t1 = min(t0 + p.seg_len, len);
    const float g = p.g[h];
    const int z0 = zt * ZW, c0 = z0 + wave * 32;           // this wave's columns
    const bool live = c0 < p.dz;
    // token t is row t, or from the end; this thread's vectors of the three
    // tiles, and how far they move from chunk to chunk
    const int64_t dir = p.rev ? -1 : 1, first = p.rev ? len - 1 - t0 : t0;
    struct At { const char* p; int row, c, at; };
    At ax[STATE ? 1 : NX], ay[NX], az[NZ];
    // (a row's last vector ends with the row: one that would pass the end is
    // moved back over the one before it, whole ones past it are not kept)
    auto place = [&](At& a, const void* base, const int64_t (&st)[3], int v, int per, int col0, int d) {
        if (v >= CH * per) v -= NTH;   // past the tile: the vector before once more
        a.row = v / per;
        a.c = col0 + v % per * 8;
        a.at = min(a.c, max(d - 8, 0));
        a.p = (const char*)base + (b * st[0] + h * st[1] + (first + dir * a.row) * st[2] + a.at) * ES;
    };
#pragma unroll
    for (int i = 0; i < NX; ++i) {
        if constexpr (!STATE) place(ax[i], p.X, p.sx, i * NTH + tid, DX / 8, 0, p.dx);
        place(ay[i], p.Y, p.sy, i * NTH + tid, DX / 8, 0, p.dx);
    }
#pragma unroll
    for (int i = 0; i < NZ; ++i) place(az[i], p.Z, p.sz, i * NTH + tid, ZW / 8, z0, p.dz);
    const int64_t mx = dir * CH * p.sx[2] * ES, my = dir * CH * p.sy[2] * ES, mz = dir * CH * p.sz[2] * ES;

    Vec8<E> rx[AHEAD && !STATE ? NX : 1], ry[AHEAD ? NX : 1], rz[AHEAD ? NZ : 1];
    // Loads of a chunk with `left` tokens carry no condition that their values
    // would have to wait for: rows behind the end read the chunk's first row
    // and are put aside when they are stored.  Rows of fewer than eight
    // elements go one by one.
    auto load_v = [&](Vec8<E>& r, At& a, int64_t move, int64_t step, int d, int left) __attribute__((always_inline)) {
        const char* q = a.p;
        if (left < CH && a.row >= left) q -= (int64_t)a.row * step;
        if constexpr (VEC) r.load8(q);
        else if (d >= 8) r.load8(q);
        else r.load(q, a.c == 0 ? d : 0);
        a.p += move;
    };
    const int64_t qx = dir * p.sx[2] * ES, qy = dir * p.sy[2] * ES, qz = dir * p.sz[2] * ES;
    auto load_x = [&](Vec8<E>& r, int i, int left) __attribute__((always_inline)) {
        load_v(r, ax[STATE ? 0 : i], mx, qx, p.dx, left);
    };
    auto load_y = [&](Vec8<E>& r, int i, int left) __attribute__((always_inline)) {
        load_v(r, ay[i], my, qy, p.dx, left);
    };
    auto load_z = [&](Vec8<E>& r, int i, int left) __attribute__((always_inline)) { load_v(r, az[i], mz, qz, p.dz, left); };
    auto load = [&](int tc) __attribute__((always_inline)) {
        if constexpr (AHEAD) {
            auto all = [&](int left) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < NX; ++i) {
                    load_y(ry[i], i, left);
                    if constexpr (!STATE) load_x(rx[i], i, left);
                }
#pragma unroll
                for (int i = 0; i < NZ; ++i) load_z(rz[i], i, left);
            };
            if (t1 - tc >= CH) all(CH);
            else all(t1 - tc);
        }
    };
    // a vector's terms into its tile, with zeros past the rows' and the chunk's ends
    const bool whole_x = VEC && p.dx == DX, whole_z = VEC && z0 + ZW <= p.dz;
    auto put = [&](Vec8<E>& r, const At& a, int col0, int d, int left, uint16_t* row, int plane, bool whole) __attribute__((always_inline)) {
        if (!whole || left < CH)
            if (a.c >= d || a.row >= left) r.zero();
        u4 t[T];
        const bool ok = terms_of(r, t);
        uint16_t* to = row + (a.c - col0);
#pragma unroll
        for (int n = 0; n < T; ++n, to += plane) {
            if constexpr (VEC) {
                *(u2*)to = u2{t[n].x, t[n].y};             // (rows keep 8 bytes, not 16)
                *(u2*)(to + 4) = u2{t[n].z, t[n].w};
            } else {
                // a last vector that was moved back starts in the one before it
                const int skip = a.c < d ? a.c - a.at : 0;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e >= skip) to[e - skip] = (uint16_t)(t[n][e >> 1] >> (16 * (e & 1)));
                for (int e = 8 - skip; e < 8; ++e) to[e] = 0;
            }
        }
        return ok;
    };
    auto stage = [&](int tc, int buf, int par) __attribute__((always_inline)) {
        const int left = t1 - tc;
#pragma unroll
        for (int i = 0; i < NX; ++i) {
            if constexpr (!AHEAD) {
                load_y(ry[0], i, left);
                if constexpr (!STATE) load_x(rx[0], i, left);
            }
            put(ry[AHEAD ? i : 0], ay[i], 0, p.dx, left, &Ys[buf][0][ay[i].row][0], CH * DXP, whole_x);
            if constexpr (!STATE) put(rx[AHEAD ? i : 0], ax[i], 0, p.dx, left, &Xs[buf][0][ax[i].row][0], CH * DXP, whole_x);
        }
        bool ok = true;
#pragma unroll
        for (int i = 0; i < NZ; ++i) {
            if constexpr (!AHEAD) load_z(rz[0], i, left);
            ok = put(rz[AHEAD ? i : 0], az[i], z0, p.dz, left, &Zs[buf][0][az[i].row][0], CH * ZP, whole_z) && ok;
        }
        if (!STATE && !ok) odd[par] = tc;
    };
    if (t0 < t1) load(t0);   // (an empty sequence has no row to read)
    if (tid <= CH) pw[tid] = decay_pow(g, tid);
    // token j of a chunk of n weighs lambda^{n-1-j}, one more backwards: element
    // j + 32 - n here, zeros behind the end
    if (tid < 2 * CH) pu[tid] = tid < CH ? decay_pow(g, CH - 1 - tid + p.rev) * p.u_mul : 0.f;
    if (tid < 2) odd[tid] = -1;
    if (tid == NTH - 1) fs = factors_of(g, CH);            // (a wave that has none of the above)
    __syncthreads();
    // the state: element (a, c0 + l32) of register r of tile a / 32, a = 8 (r / 4) + 4 hh + r % 4
    f16x S[AT];
    const int64_t state = (int64_t)bh * p.dx * p.dz;
    const int64_t frag = ((((int64_t)bh * p.nz + zt) * p.nseg + seg) * W + wave) * (AT * 4 * 256) + lane * 4;
    const int ra = p.s_t ? 1 : p.dz, rc = p.s_t ? p.dx : 1;   // S0 and SE: strides of a and c
    if (!STATE && p.nseg > 1 && !p.prefix) {
        if (p.u_waves) {
            // the states of another recurrence, whose rows are these columns
            const float* u = p.U + ((int64_t)bh * p.u_nz * p.nseg + seg) * p.u_waves * p.u_at * 1024;
            const int64_t per_zt = (int64_t)p.nseg * p.u_waves * p.u_at * 1024;
            const int c = c0 + l32, row = (c >> 5) * 1024 + ((c >> 3) & 3) * 256 + ((c >> 2) & 1) * 128 + (c & 3);
#pragma unroll
            for (int k = 0; k < AT; ++k)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int a = 32 * k + 8 * (r >> 2) + 4 * hh + (r & 3), w = a >> 5;
                    S[k][r] = a < p.dx && c < p.dz
                                  ? u[w / p.u_waves * per_zt + (int64_t)(w % p.u_waves) * p.u_at * 1024 + row + (a & 31) * 4] : 0.f;
                }
        } else {
#pragma unroll
            for (int k = 0; k < AT * 4; ++k) {
                const f4 v = *(const f4*)(p.U + frag + k * 256);
#pragma unroll
                for (int e = 0; e < 4; ++e) S[k / 4][(k % 4) * 4 + e] = v[e];
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < AT; ++k)
#pragma unroll
            for (int r = 0; r < 16; ++r) S[k][r] = 0.f;
        if (!STATE && p.S0) {
#pragma unroll
            for (int k = 0; k < AT; ++k)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int a = 32 * k + 8 * (r >> 2) + 4 * hh + (r & 3), c = c0 + l32;
                    if (a < p.dx && c < p.dz) S[k][r] = p.S0[state + (int64_t)a * ra + (int64_t)c * rc];
                }
        }
        // few and small states: each segment adds up those before it, which
        // saves the scan
        if (!STATE && p.prefix && live) {
            Factors of_segments = for_wave(factors_of(g, p.seg_len));
            for (int t = 0; t < seg; ++t) {
                const float lam = of_segments.next();
                const float* u = p.U + frag - (int64_t)(seg - t) * W * (AT * 4 * 256);
#pragma unroll
                for (int k = 0; k < AT * 4; ++k) {
                    const f4 v = *(const f4*)(u + k * 256);
#pragma unroll
                    for (int e = 0; e < 4; ++e) S[k / 4][(k % 4) * 4 + e] = S[k / 4][(k % 4) * 4 + e] * lam + v[e];
                }
            }
        }
    }
    // weights of this lane: of scores (token l32, tokens j of its registers) and
    // of the state's part of token l32
    float wp[STATE ? 1 : 16], wq = 0.f;
    if constexpr (!STATE) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int j = 8 * (r >> 2) + 4 * hh + (r & 3);
            wp[r] = j <= l32 ? pw[l32 - j] * p.p_mul : 0.f;
        }
        wq = pw[l32 + 1 - p.rev] * p.q_mul;
    }
    // this lane's row of the output: token l32, or from the end
    char* orow = (char*)p.O + (b * p.so[0] + h * p.so[1] + (first + dir * l32) * p.so[2]) * ES;
    const int64_t mo = dir * CH * p.so[2] * ES;
    Factors of_chunks = for_wave(fs);

    for (int tc = t0, par = 0; tc < t1; tc += CH, par ^= 1) {
        const int buf = NB == 2 ? par : 0;
        stage(tc, buf, par);
        __syncthreads();
        if (tc + CH < t1) load(tc + CH);
        const int cnt = min(CH, t1 - tc);
        if (live) {
            const bool rest = odd[par] == tc;
            // Fragments are read a step ahead of the products that take them, held
            // there by scheduling barriers: left alone, the reads sink to their uses.
            // Z^T: this wave's columns, tokens of the update's and the scores' order
            b8 z[2][T];
            auto read_z = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int n = 0; n < T; ++n) {
                        const int c = wave * 32 + (lane & 16) + 4 * (lane & 3), j = 16 * s + 4 * hh + ((lane & 15) >> 2);
                        z[s][n] = join(read_tr(&Zs[buf][n][j][c]), read_tr(&Zs[buf][n][j + 8][c]));
                    }
            };
            // Y^T: rows a of tiles 2 (i / 2) and the one after it, tokens of half i % 2
            b8 yt[2][2][T];
            auto read_yt = [&](int i) __attribute__((always_inline)) {
                const int c = 64 * (i >> 1) + (lane & 16) + 4 * (lane & 3), j = 16 * (i & 1) + 4 * hh + ((lane & 15) >> 2);
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (2 * (i >> 1) + k < AT) {
#pragma unroll
                        for (int n = 0; n < T; ++n)
                            yt[i & 1][k][n] = join(read_tr(&Ys[buf][n][j][c + 32 * k]), read_tr(&Ys[buf][n][j + 8][c + 32 * k]));
                    }
            };
            const float wc = cnt == CH ? of_chunks.next() : pw[cnt];
            f16x P{}, O{};
            if constexpr (!STATE) {
                b8 x[2][T], y[2][T];
                auto read_xy = [&](int ks) __attribute__((always_inline)) {
                    const int c = 16 * ks + 4 * hh;
#pragma unroll
                    for (int n = 0; n < T; ++n) {
                        x[ks & 1][n] = join(*(const s4*)&Xs[buf][n][l32][c], *(const s4*)&Xs[buf][n][l32][c + 8]);
                        y[ks & 1][n] = join(*(const s4*)&Ys[buf][n][l32][c], *(const s4*)&Ys[buf][n][l32][c + 8]);
                    }
                };
                read_xy(0);
#pragma unroll
                for (int ks = 0; ks < DX / 16; ++ks) {
                    if (ks + 1 < DX / 16) read_xy(ks + 1);
                    else read_z();
                    __builtin_amdgcn_sched_barrier(0);
                    b8 st[NS];
                    float sv[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        sv[e] = S[ks / 2][8 * (ks & 1) + e];
                        S[ks / 2][8 * (ks & 1) + e] = sv[e] * wc;   // the chunk's decay, for its update below
                    }
                    split8<NS>(sv, st);
                    mma2<T, T, T, NS, T, MS>(P, y[ks & 1], x[ks & 1], O, st, x[ks & 1]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
                read_z();
            }
            read_yt(0);
            // (read here: the powers' words cost less than registers that keep them)
            float wu[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) wu[r] = pu[8 * (r >> 2) + 4 * hh + (r & 3) + CH - cnt];
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (!STATE) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    O[r] *= wq;
                    // put aside, not multiplied: a later token's NaN stays its own
                    P[r] = 8 * (r >> 2) + 4 * hh + (r & 3) <= l32 ? P[r] * wp[r] : 0.f;
                }
                if (!rest) {
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        b8 pt[NS];
                        float pv[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) pv[e] = P[8 * s + e];
                        split8<NS>(pv, pt);
                        mma<T, NS, MS>(O, z[s], pt);
                    }
                } else {
                    // 0 times an infinity or NaN of a later token would reach
                    // earlier ones: token by token, only those that are seen
#pragma unroll
                    for (int rj = 0; rj < 16; ++rj)
#pragma unroll 1
                        for (int hj = 0; hj < 2; ++hj) {
                            const int j = 8 * (rj >> 2) + 4 * hj + (rj & 3);
                            const float pj = __shfl(P[rj], l32 + 32 * hj);
#pragma unroll
                            for (int r = 0; r < 16; ++r) {
                                const int c = wave * 32 + 8 * (r >> 2) + 4 * hh + (r & 3);
                                float zv = 0.f;
#pragma unroll
                                for (int n = T - 1; n >= 0; --n) zv += __uint_as_float((uint32_t)Zs[buf][n][j][c] << 16);
                                if (j <= l32) O[r] += pj * zv;
                            }
                        }
                }
                Out4<E> o[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float v[4] = {O[4 * q], O[4 * q + 1], O[4 * q + 2], O[4 * q + 3]};
                    o[q] = round4((E*)nullptr, v);
                }
                if constexpr (ES == 2) {
                    // the halves of a wave hold columns 0..3 and 4..7 of every
                    // eight: they trade, so that a lane stores eight at once
#pragma unroll
                    for (int q = 0; q < 4; q += 2)
#pragma unroll
                        for (int w = 0; w < 2; ++w) {
                            const auto r = __builtin_amdgcn_permlane32_swap(o[q].w[w], o[q + 1].w[w], false, false);
                            o[q].w[w] = r[0];
                            o[q + 1].w[w] = r[1];
                        }
                    if (l32 < cnt) {
#pragma unroll
                        for (int q = 0; q < 4; q += 2) {
                            const int c = c0 + 8 * (q + hh);
                            if (c + 8 <= p.dz) {
                                *(u4u*)(orow + c * ES) = u4{o[q].w[0], o[q].w[1], o[q + 1].w[0], o[q + 1].w[1]};
                            } else {
                                store4<E>(orow, c, p.dz, o[q]);
                                store4<E>(orow, c + 4, p.dz, o[q + 1]);
                            }
                        }
                    }
                } else if (l32 < cnt) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) store4<E>(orow, c0 + 8 * q + 4 * hh, p.dz, o[q]);
                }
                orow += mo;
            }
            b8 wz[2][kStateTerms];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                float zv[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float v = (float)z[s][T - 1][e];
#pragma unroll
                    for (int n = T - 2; n >= 0; --n) v += (float)z[s][n][e];
                    zv[e] = v * wu[8 * s + e];
                }
                split8<kStateTerms>(zv, wz[s]);
            }
            if constexpr (STATE) {
#pragma unroll
                for (int k = 0; k < AT; ++k)
#pragma unroll
                    for (int r = 0; r < 16; ++r) S[k][r] *= wc;
            }
            constexpr int STEPS = 2 * ((AT + 1) / 2);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                if (i + 1 < STEPS) read_yt(i + 1);
                __builtin_amdgcn_sched_barrier(0);
                const int k = 2 * (i >> 1);
                if (k + 1 < AT)
                    mma2<T, kStateTerms, kStateTerms, T, kStateTerms, kStateTerms>(S[k + 1 < AT ? k + 1 : 0], yt[i & 1][1], wz[i & 1],
                                                                                   S[k], yt[i & 1][0], wz[i & 1]);
                else
                    mma<T, kStateTerms, kStateTerms>(S[k], yt[i & 1][0], wz[i & 1]);
            }
        }
        // two buffers: the next chunk's barrier says that everybody has left
        // the one that is written after it
        if constexpr (NB == 1) __syncthreads();
    }

    if (!live) return;
    if constexpr (STATE) {
#pragma unroll
        for (int k = 0; k < AT * 4; ++k) {
            f4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = S[k / 4][(k % 4) * 4 + e];
            *(f4*)(p.U + frag + k * 256) = v;
        }
    } else if (p.SE && t1 == len) {
#pragma unroll
        for (int k = 0; k < AT; ++k)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int a = 32 * k + 8 * (r >> 2) + 4 * hh + (r & 3), c = c0 + l32;
                if (a < p.dx && c < p.dz) p.SE[state + (int64_t)a * ra + (int64_t)c * rc] = S[k][r];
            }
    }
}

// The segments' own states, in the accumulators' order, become the states
// before them: P_0 = S0, P_{s+1} = lambda^{seg_len} P_s + U_s.  A thread takes
// four elements through all segments.
__global__ __launch_bounds__(256) void k_lin_scan(const LinParams p) {
    const int waves = p.waves, at = p.at;
    const int64_t per = (int64_t)waves * at * 256;         // four-element groups of a segment's tile
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= per * p.nz * p.B * p.H) return;
    const int64_t tile = i / per;
    const int e = (int)(i % per), lane = e & 63, grp = (e >> 6) % (at * 4), wave = (e >> 6) / (at * 4);
    const int zt = (int)(tile % p.nz), bh = (int)(tile / p.nz), b = bh / p.H, h = bh - b * p.H;
    const int c = (zt * waves + wave) * 32 + (lane & 31), a0 = 32 * (grp >> 2) + 8 * (grp & 3) + 4 * (lane >> 5);
    if (c >= p.dz) return;
    const int len = p.lens ? min(max(p.lens[b], 0), p.L) : p.L;
    Factors of_segments = factors_of(p.g[h], p.seg_len);   // (those of the chunks' launch: the same bits as without a scan)
    const int ra = p.s_t ? 1 : p.dz, rc = p.s_t ? p.dx : 1;
    f4 cur;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        cur[k] = p.S0 && a0 + k < p.dx ? p.S0[(int64_t)bh * p.dx * p.dz + (int64_t)(a0 + k) * ra + (int64_t)c * rc] : 0.f;
    float* u = p.U + (tile * p.nseg * per + e) * 4;
    // every segment with tokens gets its start, segment 0 too: the state may
    // be updated in place, so the chunks never read S0 beside its writer.
    // Eight segments are asked for at a time (against one after the other, us:
    // 18 states of 64 x 64, 16 segments 8.8 -> 5.3, 64 of 96 x 80 7.7 -> 7.0, 64
    // of 128 x 128 12.7 -> 14).
    const int n = max(1, (int)(((int64_t)len + p.seg_len - 1) / p.seg_len));
    constexpr int AT_ONCE = 8;
    for (int s0 = 0; s0 < n; s0 += AT_ONCE) {
        f4 v[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) v[k] = s0 + k + 1 < n ? *(const f4*)(u + (s0 + k) * per * 4) : f4{};
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
            if (s0 + k < n) {
                *(f4*)(u + (s0 + k) * per * 4) = cur;
                const float lam = of_segments.next();
#pragma unroll
                for (int e = 0; e < 4; ++e) cur[e] = cur[e] * lam + v[k][e];
            }
    }
}

// One token: S <- lambda S + k^T v, o = scale q S, in one pass over S, which
// bounds it (read and written once; 2048 states of 128 x 128 57 us, 4.75 TB/s,
// what a copy of as many bytes reaches).  A workgroup takes COLS columns of a
// head's state; a thread four of them and every (256 / (COLS / 4))-th row.
template <class E>
__device__ __forceinline__ float load1(const void* p, int64_t i);
template <>
__device__ __forceinline__ float load1<float>(const void* p, int64_t i) { return ((const float*)p)[i]; }
template <>
__device__ __forceinline__ float load1<Half>(const void* p, int64_t i) { return (float)((const _Float16*)p)[i]; }
template <>
__device__ __forceinline__ float load1<Bf16>(const void* p, int64_t i) {
    return __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16);
}

template <class E, int COLS>
__global__ __launch_bounds__(256) void k_lin_step(const LinStepParams p) {
    constexpr int CT = COLS / 4, RT = 256 / CT;
    __shared__ float ks[256], qs[256];
    __shared__ __align__(16) float part[RT][COLS + 4];
    const int tid = threadIdx.x, ct = tid % CT, rt = tid / CT;
    const int ntile = (p.dv + COLS - 1) / COLS;
    const int64_t bh = blockIdx.x / ntile;
    const int c = (blockIdx.x % ntile) * COLS + 4 * ct;
    const int64_t b = bh / p.H, h = bh - b * p.H;
    float* S = p.S + bh * p.dk * p.dv;
    // full vectors where rows keep their 16 bytes, else element by element
    const bool vec = p.dv % 4 == 0 && ((uintptr_t)p.S & 15) == 0;
    const Decay lam = decay_of(p.g[h]);
    if (tid < p.dk) {
        ks[tid] = load1<E>(p.k, b * p.sk[0] + h * p.sk[1] + tid);
        qs[tid] = load1<E>(p.q, b * p.sq[0] + h * p.sq[1] + tid) * p.scale;
    }
    float v[4], o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = c + e < p.dv ? load1<E>(p.v, b * p.sv[0] + h * p.sv[1] + c + e) : 0.f;
    __syncthreads();
    if (c < p.dv) {
        if (vec) {
#pragma unroll 8
            for (int a = rt; a < p.dk; a += RT) {
                f4 s = *(const f4*)(S + (int64_t)a * p.dv + c);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[e] = lam.of(s[e], ks[a] * v[e]);
                    o[e] += qs[a] * s[e];
                }
                *(f4*)(S + (int64_t)a * p.dv + c) = s;
            }
        } else {
            for (int a = rt; a < p.dk; a += RT)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e < p.dv) {
                        const float s = lam.of(S[(int64_t)a * p.dv + c + e], ks[a] * v[e]);
                        S[(int64_t)a * p.dv + c + e] = s;
                        o[e] += qs[a] * s;
                    }
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) part[rt][4 * ct + e] = o[e];
    __syncthreads();
    if (tid < CT) {
        float r[4] = {0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < RT; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] += part[k][4 * tid + e];
        store4<E>((char*)p.o + (b * p.so[0] + h * p.so[1]) * (int64_t)(sizeof(Vec8<E>) / 8), c, p.dv, round4((E*)nullptr, r));
    }
}

// ===========================================================================
// Builders
// ===========================================================================
LinShape lin_shape(int32_t type, int64_t B, int64_t H, int64_t L, int64_t dx, int64_t dz) {
    LinShape s{};
    // head sizes that are no multiple of eight take the larger kernels
    s.vec = dx % 8 == 0 && dz % 8 == 0;
    s.dxp = dx <= 64 && s.vec ? 64 : dx <= 96 && s.vec ? 96 : dx <= 128 ? 128 : 256;
    // (two waves: nothing idles at 64 columns; bf16, 2 / 4 waves, us: 128 heads x
    // 2048 x 64 55 / 69, 256 heads 83 / 104; fp32 138 / 130 and 250 / 220)
    s.waves = dz <= 64 && s.vec ? 2 : 4;
    s.nz = (int32_t)((dz + 32 * s.waves - 1) / (32 * s.waves));
    // Sequences are cut where the heads alone leave more than half of the chip
    // without work: into segments for two waves a SIMD, of at least five chunks
    // (two where a chunk takes several products for one), since the other
    // two launches cost some 10 us and a chunk 1 to 3 (us at 1, 2, 4, ..
    // segments: 16 heads x 2048 x 128 bf16 144, 122, 73, 8: 53, 11: 44, 16: 47;
    // 128 heads x 4000 x 64 192, 157, 116, 8: 88, 12: 103; 16 heads x 512 x 64
    // fp16 49, 47, 32, 8: 26, 16: 28; 256 heads x 2000 x 128 176, 214, 246;
    // 128 heads x 300 x 64 24, 30, 30)
    const int64_t wgs = B * H * s.nz, chunks = (L + CH - 1) / CH, want = s.waves == 4 ? 512 : 1024;
    int64_t nseg = 1;
    if (2 * wgs < want && chunks >= 12) nseg = std::max<int64_t>(std::min((want + wgs - 1) / wgs, chunks / (type == FT_BF16 ? 5 : 2)), 1);
    const int64_t per = std::max<int64_t>((chunks + nseg - 1) / nseg, 1);
    s.nseg = (int32_t)std::max<int64_t>((chunks + per - 1) / per, 1);
    s.seg_len = (int32_t)(per * CH);
    s.u_floats = s.nseg > 1 ? (int64_t)s.nseg * wgs * s.waves * 32 * s.dxp : 0;
    return s;
}

void build_lin(int32_t type, const LinShape& s, const LinParams& p0, bool state_only, LaunchRec* rec) {
    LinParams p = p0;
    p.nseg = s.nseg;
    p.seg_len = s.seg_len;
    p.nz = s.nz;
    rec->grid = dim3((unsigned)((int64_t)p.B * p.H * s.nz * s.nseg), 1, 1);
    rec->block = dim3(64 * s.waves, 1, 1);
    rec->name = state_only ? "lin_state" : "lin_chunks";
#define QX_K(E, D, W, V) rec->fn = state_only ? (const void*)k_lin<E, D, W, true, V> : (const void*)k_lin<E, D, W, false, V>;
#define QX_D(E)                                                             \
    if (!s.vec) {                                                           \
        if (s.dxp == 128) { QX_K(E, 128, 4, false) }                        \
        else { QX_K(E, 256, 4, false) }                                     \
    } else if (s.waves == 2) {                                              \
        if (s.dxp == 64) { QX_K(E, 64, 2, true) }                           \
        else if (s.dxp == 96) { QX_K(E, 96, 2, true) }                      \
        else if (s.dxp == 128) { QX_K(E, 128, 2, true) }                    \
        else { QX_K(E, 256, 2, true) }                                      \
    } else {                                                                \
        if (s.dxp == 64) { QX_K(E, 64, 4, true) }                           \
        else if (s.dxp == 96) { QX_K(E, 96, 4, true) }                      \
        else if (s.dxp == 128) { QX_K(E, 128, 4, true) }                    \
        else { QX_K(E, 256, 4, true) }                                      \
    }
    if (type == FT_F32) { QX_D(float) }
    else if (type == FT_F16) { QX_D(Half) }
    else { QX_D(Bf16) }
#undef QX_D
#undef QX_K
    rec->set_params(p);
}

void build_lin_scan(const LinShape& s, const LinParams& p0, LaunchRec* rec) {
    LinParams p = p0;
    p.nseg = s.nseg;
    p.seg_len = s.seg_len;
    p.nz = s.nz;
    p.waves = s.waves;
    p.at = s.dxp / 32;
    const int64_t n = (int64_t)s.waves * (s.dxp / 32) * 256 * s.nz * p.B * p.H;
    rec->fn = (const void*)k_lin_scan;
    rec->grid = dim3((unsigned)((n + 255) / 256), 1, 1);
    rec->block = dim3(256, 1, 1);
    rec->name = "lin_scan";
    rec->set_params(p);
}

void build_lin_step(const LinStepParams& p0, LaunchRec* rec) {
    LinStepParams p = p0;
    // whole rows of the state (512 bytes at dv 128) once there are two heads
    // for every CU, else 32 columns a workgroup (32 / 128 columns, us, states
    // of 128 x 128: 16 heads 4.1 / 5.4, 256 heads 7.4 / 9.1, 512 heads 12.4 /
    // 10.7, 1024 heads 23.7 / 22.5)
    p.cols = (int64_t)p.B * p.H >= 512 ? 128 : 32;
    const int64_t tiles = (p.dv + p.cols - 1) / p.cols;
    rec->grid = dim3((unsigned)((int64_t)p.B * p.H * tiles), 1, 1);
    rec->block = dim3(256, 1, 1);
    rec->name = "lin_step";
#define QX_K(E) rec->fn = p.cols == 128 ? (const void*)k_lin_step<E, 128> : (const void*)k_lin_step<E, 32>;
    if (p.type == FT_F32) { QX_K(float) }
    else if (p.type == FT_F16) { QX_K(Half) }
    else { QX_K(Bf16) }
#undef QX_K
    rec->set_params(p);
}

}  // namespace qx
