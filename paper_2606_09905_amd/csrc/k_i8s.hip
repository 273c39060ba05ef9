// k_i8s.hip -- products of 8-bit operands with a scale for each token and
// each output channel, and the quantisation of tokens to such operands.
//
//   Y[m][n] = sa[m] sw[n] sum_k A[m][k] W[n][k] + bias[n]
//
// The sum is exact in int32 (|sum| <= 128^2 K < 2^31 for K < 2^17); scales and
// bias are applied in fp32 and the result rounded once to Y's type.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "qx_internal.h"

namespace qx {

namespace {

typedef int i4 __attribute__((ext_vector_type(4)));
typedef int i4u __attribute__((ext_vector_type(4), aligned(1)));
typedef int i16x __attribute__((ext_vector_type(16)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef u4 u4u __attribute__((aligned(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef f4 f4u __attribute__((aligned(4)));

struct Half { uint16_t v; };
struct Bf16 { uint16_t v; };

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(Half x) { return (float)__builtin_bit_cast(_Float16, x.v); }
__device__ __forceinline__ float to_f(Bf16 x) { return __uint_as_float((uint32_t)x.v << 16); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(Half* p, float v) { p->v = __builtin_bit_cast(uint16_t, (_Float16)v); }
__device__ __forceinline__ void put(Bf16* p, float v) { p->v = __builtin_bit_cast(uint16_t, (__bf16)v); }

// eight elements of a row from column c on, zeros past `cols`, at any address
template <class E>
__device__ __forceinline__ void load8(const E* row, int64_t c, int64_t cols, float (&x)[8]) {
    if (c + 8 <= cols) {
        if constexpr (sizeof(E) == 4) {
            const f4 a = *(const f4u*)(row + c), b = *(const f4u*)(row + c + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
        } else {
            const u4 v = *(const u4u*)(row + c);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = to_f(E{(uint16_t)v[i]});
                x[2 * i + 1] = to_f(E{(uint16_t)(v[i] >> 16)});
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = c + i < cols ? to_f(row[c + i]) : 0.f;
    }
}

// |x| as an integer: orders like the value, with infinities and NaN above all
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// A sum's result: its row's scale, then its channel's, then the bias.  The
// first product may pass fp32's range where the result does not: then the
// channel's scale, which is below one, goes first.  (A sum is below 2^31, so
// that takes a row's scale of at least kLargeScale.)
constexpr float kLargeScale = 0x1p97f;
__device__ __forceinline__ float scaled(int sum, float sa, float sw, float bias) {
    const float t = (float)sum * sa;
    return fabsf(t) == __builtin_inff() ? __builtin_fmaf((float)sum * sw, sa, bias) : __builtin_fmaf(t, sw, bias);
}

// scale of a row whose largest magnitude is m; NaN for infinities and NaN
__device__ __forceinline__ float scale_of(uint32_t m) {
    return m >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : __uint_as_float(m) / 127.f;
}
__device__ __forceinline__ uint32_t quant4(const float* x, float s) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // (a subnormal scale is coarse: the quotient may pass 127)
        const int q = (int)fminf(fmaxf(rintf(x[i] / s), -127.f), 127.f);
        w |= ((uint32_t)q & 0xFFu) << (8 * i);
    }
    return w;
}

}  // namespace

// sixteen bytes of a row from k on, at any address, zeros past K: the row's
// last sixteen shifted down where they end inside the piece (rows shorter than
// that go byte by byte)
__device__ __forceinline__ i4 load16(const int8_t* row, int k, int K) {
    if (K >= 16) {
        const int at = min(k, K - 16), over = k - at;      // bytes of the piece past K
        const i4 v = *(const i4u*)(row + at);
        uint64_t lo = (uint32_t)v[0] | (uint64_t)(uint32_t)v[1] << 32, hi = (uint32_t)v[2] | (uint64_t)(uint32_t)v[3] << 32;
        const int sh = 8 * (over & 7);
        if (over & 8) {
            lo = hi;
            hi = 0;
        }
        lo = sh ? lo >> sh | hi << (64 - sh) : lo;
        hi >>= sh;
        if (over >= 16) lo = hi = 0;
        return i4{(int)lo, (int)(lo >> 32), (int)hi, (int)(hi >> 32)};
    }
    i4 v{};
#pragma unroll
    for (int i = 0; i < 15; ++i)
        if (k + i < K) v[i >> 2] |= (int)((uint32_t)(uint8_t)row[k + i] << (8 * (i & 3)));
    return v;
}

// WPR waves of a workgroup's four take a row: its largest magnitude, then the
// quotients.  A row stays in registers where it fits (NV vectors a lane);
// longer ones are read again, from L2.  Bound by reading x once: 8192 x 4096
// bf16 23.7 us, 4.2 TB/s read and written.
// The workgroups behind them copy 8-bit weights (wsrc) into rows of ldq bytes.
template <class E, int WPR>
__global__ __launch_bounds__(256) void k_quant_i8(const QuantI8Params p) {
    constexpr int NV = 4, LPR = 64 * WPR;
    __shared__ uint32_t wm[4];
    const int tid = threadIdx.x, wave = tid >> 6, l = tid % LPR;
    if ((int)blockIdx.x >= p.row_blocks) {
        const int64_t per = p.ldq / 16, n = per * p.wrows;
        for (int64_t i = (int64_t)(blockIdx.x - p.row_blocks) * 256 + tid; i < n; i += (int64_t)(gridDim.x - p.row_blocks) * 256) {
            const int64_t r = i / per;
            *(i4*)(p.wdst + i * 16) = load16(p.wsrc + r * p.cols, (int)(i - r * per) * 16, (int)p.cols);
        }
        return;
    }
    const int64_t row = (int64_t)blockIdx.x * (4 / WPR) + wave / WPR;
    const bool live = row < p.rows;
    const E* x = (const E*)p.x + (live ? row : 0) * p.ld;
    float v[NV][8];
    uint32_t m = 0;
    if (live) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t c = ((int64_t)k * LPR + l) * 8;
            if (c < p.cols) {
                load8(x, c, p.cols, v[k]);
#pragma unroll
                for (int i = 0; i < 8; ++i) m = max(m, mag(v[k][i]));
            }
        }
        for (int64_t c = ((int64_t)NV * LPR + l) * 8; c < p.cols; c += (int64_t)LPR * 8) {
            float t[8];
            load8(x, c, p.cols, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, mag(t[i]));
        }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    if constexpr (WPR == 4) {
        if ((tid & 63) == 0) wm[wave] = m;
        __syncthreads();
        m = max(max(wm[0], wm[1]), max(wm[2], wm[3]));
    }
    if (!live) return;
    const float s = scale_of(m);
    const bool zero = !(s > 0.f);   // a row of zeros, or one whose scale is NaN
    if (l == 0) p.scale[row] = s;
    int8_t* q = p.q + row * p.ldq;
    const bool vec = ((uintptr_t)q & 7) == 0;
    auto store = [&](int64_t c, const float (&t)[8]) {
        const uint32_t a = zero ? 0u : quant4(t, s), b = zero ? 0u : quant4(t + 4, s);
        if (vec && c + 8 <= p.ldq) {
            *(uint2*)(q + c) = make_uint2(a, b);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < p.ldq) q[c + i] = (int8_t)((i < 4 ? a : b) >> (8 * (i & 3)));
        }
    };
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int64_t c = ((int64_t)k * LPR + l) * 8;
        if (c < p.cols) store(c, v[k]);
    }
    const float none[8] = {};
    for (int64_t c = (int64_t)l * 8; c < p.ldq; c += (int64_t)LPR * 8) {
        if (c >= p.cols) {
            store(c, none);
        } else if (c >= (int64_t)NV * LPR * 8) {
            float t[8];
            load8(x, c, p.cols, t);
            store(c, t);
        }
    }
}

__device__ const i4 g_zero16{};

// A wait for all but the n newest of a wave's loads.
template <int N>
__device__ __forceinline__ void wait_loads() {
    static_assert(N <= 63, "counter range");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0F70);
}

// BM x BN tiles, WM x WN waves, K in tiles of 128 bytes through a ring of
// STAGES.  Bound by the matrix cores and their power at 256 x 256 (8192^3 541
// us, 2030 TOPS; without its loads 386, without its LDS reads 522, the products
// alone 421): spreading the loads over the products, by halves of the waves
// too, fragments read a step ahead through a ring of four 64-byte tiles, and
// four waves of 128 x 128 all measured 525 to 650.  ALIGNED: rows start at
// 16-byte addresses and go to LDS directly, STAGES - 1 tiles ahead; else
// through registers, two ahead.
template <class E, int BM, int BN, int WM, int WN, int STAGES, bool ALIGNED>
__global__ __launch_bounds__(64 * WM * WN) void k_gemm_i8s(const GemmI8sParams p) {
    constexpr int NW = WM * WN, NTH = 64 * NW, BK = 128, KC = BK / 16;
    constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int LA = BM * KC / NTH, LB = BN * KC / NTH, LPT = LA + LB, CH = (BM + BN) * KC;
    static_assert(LA * NTH == BM * KC && LB * NTH == BN * KC, "whole loads");
    __shared__ i4 St[STAGES][CH];
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
    int pid = blockIdx.x;
    const int total = gridDim.x;
    // consecutive workgroups go to the eight XCDs in turn: each XCD takes a
    // contiguous run of tiles, whose panels share its L2
    {
        const int per = total >> 3, rest = total & 7, x = pid & 7, i = pid >> 3;
        pid = x * per + min(x, rest) + i;
    }
    constexpr int GR = 8;
    const int per_group = GR * p.tiles_n, gid = pid / per_group, first_m = gid * GR;
    const int gsz = min(p.tiles_m - first_m, GR), in = pid - gid * per_group;
    const int m0 = (first_m + in % gsz) * BM, n0 = in / gsz * BN;

    // this thread's pieces of a tile: a row's 16 bytes at place c of 8, kept at
    // place c ^ (row / 2 % 8): two rows fill the 64 banks, and sixteen rows of a
    // read lie in sixteen different places of them
    const int8_t* src[LPT];
    int sk[LPT];
#pragma unroll
    for (int i = 0; i < LPT; ++i) {
        const int q = (i < LA ? i : i - LA) * NTH + tid, row = q / KC;
        src[i] = i < LA ? p.A + (int64_t)min(m0 + row, p.M - 1) * p.lda : p.W + (int64_t)min(n0 + row, p.N - 1) * p.ldw;
        sk[i] = ((q % KC) ^ (row >> 1 & 7)) * 16;
        if constexpr (ALIGNED) src[i] += sk[i];
    }
    const int kt = (p.K + BK - 1) / BK, whole = p.K / BK;
    i4 reg[2][ALIGNED ? 1 : LPT];
    auto issue = [&](int t, int set) __attribute__((always_inline)) {
        if constexpr (ALIGNED) {
            const unsigned base = (unsigned)(uintptr_t)&St[t % STAGES][0] + (unsigned)wave * 1024u;
#pragma unroll
            for (int i = 0; i < LPT; ++i) {
                const int8_t* at = src[i] + (int64_t)t * BK;
                // pieces past K (the last tile's) come from zeros
                if (t >= whole && t * BK + sk[i] >= p.K) at = (const int8_t*)&g_zero16;
                // (a load that takes its LDS address from M0 needs one wait state behind the write of M0)
                asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                             :: "v"(at), "s"(base + i * NTH * 16) : "memory", "m0");
            }
        } else {
            if (t < whole) {
#pragma unroll
                for (int i = 0; i < LPT; ++i) reg[set][i] = *(const i4u*)(src[i] + t * BK + sk[i]);
            } else {
#pragma unroll
                for (int i = 0; i < LPT; ++i) reg[set][i] = load16(src[i], t * BK + sk[i], p.K);
            }
        }
    };
    // the scales of this wave's rows, to find out whether any is large
    constexpr int LS = (BM / WM + 63) / 64;
    float rs[LS];
#pragma unroll
    for (int i = 0; i < LS; ++i) rs[i] = p.sa[min(m0 + wm * (BM / WM) + i * 64 + lane % (BM / WM), p.M - 1)];
    i16x acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = i16x{};
    auto compute = [&](const i4* S) __attribute__((always_inline)) {
#pragma unroll
        for (int ks = 0; ks < KC / 2; ++ks) {
            i4 a[TM], b[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int row = wm * (BM / WM) + i * 32 + l32;
                a[i] = S[row * KC + ((2 * ks + hh) ^ (row >> 1 & 7))];
            }
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int row = wn * (BN / WN) + j * 32 + l32;
                b[j] = S[BM * KC + row * KC + ((2 * ks + hh) ^ (row >> 1 & 7))];
            }
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[i], b[j], acc[i][j], 0, 0, 0);
        }
    };
    if constexpr (ALIGNED) {
#pragma unroll
        for (int t = 0; t < STAGES - 1; ++t)
            if (t < kt) issue(t, 0);
        for (int t = 0; t < kt; ++t) {
            // tile t has landed (the STAGES - 2 behind it may be in flight,
            // none of them near the end), everywhere past the barrier, and
            // every wave is done with the slot that is filled next
            if (t + STAGES - 2 < kt) wait_loads<(STAGES - 2) * LPT>();
            else wait_loads<0>();
            __syncthreads();
            if (t + STAGES - 1 < kt) issue(t + STAGES - 1, 0);
            compute(St[t % STAGES]);
        }
    } else {
        auto step = [&](int t, int set) __attribute__((always_inline)) {
            i4* S = St[set];
#pragma unroll
            for (int i = 0; i < LPT; ++i) S[i * NTH + tid] = reg[set][i];
            __syncthreads();
            if (t + 2 < kt) issue(t + 2, set);
            compute(S);
        };
        if (kt > 0) issue(0, 0);
        if (kt > 1) issue(1, 1);
        for (int t = 0; t < kt; t += 2) {
            step(t, 0);
            if (t + 1 < kt) step(t + 1, 1);
        }
    }
    // lane holds column l32 of a 32 x 32 block, rows 8 (r / 4) + 4 hh + r % 4
    E* Y = (E*)p.Y;
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < LS; ++i) most = fmaxf(most, fabsf(rs[i]));
    auto results = [&](auto value) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int n = n0 + wn * (BN / WN) + j * 32 + l32;
            if (n >= p.N) continue;
            const float sw = p.sw[n], bias = p.bias ? p.bias[n] : 0.f;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int m = m0 + wm * (BM / WM) + i * 32 + 8 * (r >> 2) + 4 * hh + (r & 3);
                    if (m < p.M) put(Y + (int64_t)m * p.N + n, value(acc[i][j][r], p.sa[m], sw, bias));
                }
        }
    };
    // rows so large hardly ever come: the wave looks once (8192^3 0.8% longer; for each
    // sum by itself 8192 x 8192 x 256 takes 3.5% longer)
    if (__any(most >= kLargeScale)) results(scaled);
    else results([](int sum, float sa, float sw, float bias) { return __builtin_fmaf((float)sum * sa, sw, bias); });
}

// Few rows (M <= 32): bound by reading W once, so a workgroup takes 16 NT of
// W's rows and its eight waves share K, 64 bytes of every 512 each, with UK
// such loads in flight a lane; the waves' partial sums meet in LDS.  W is the
// A operand of v_mfma_i32_16x16x64_i8, 16 tokens the B operand.
// FUSED: every workgroup quantises the rows of x itself while its first loads
// of W are in flight, which saves a launch; at most 32 elements a thread.
// (24 x 8192 x 4096 bf16 with the quantisation 15.0 us, of which reading W at
// a copy's rate takes 7 to 9.)
constexpr int kFusedRows = 16, kFusedElems = 16384;
template <class E, int MT, int NT, bool FUSED>
__global__ __launch_bounds__(512) void k_skinny_i8s(const GemmI8sParams p) {
    constexpr int UK = NT * (FUSED ? 1 : 1 + MT) <= 3 ? 8 : 4;
    extern __shared__ __align__(16) int8_t lds[];
    i4* red = (i4*)lds;                                    // [8][MT][NT][64]
    float* sa_l = (float*)(lds + 8 * MT * NT * 1024);      // FUSED: [16] scales, then the rows
    int8_t* xq = lds + 8 * MT * NT * 1024 + 64;
    const int ldq = (p.K + 15) / 16 * 16 + 16;             // rows 16 bytes apart in their banks
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, kg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n0 = blockIdx.x * (16 * NT), k0 = wave * 64 + kg * 16;

    // FUSED: a group of waves takes a row, or a wave takes two; a thread's
    // four vectors of it are asked for ahead of W
    const int wpr = p.M == 1 ? 8 : p.M == 2 ? 4 : p.M <= 4 ? 2 : 1;
    const bool two = FUSED && p.M > 8;
    const int xr = wave / wpr, xl = tid % (64 * wpr);
    float xv[FUSED ? 4 : 1][8];
    auto x_at = [&](int s, int& row, int& c) {
        row = two ? xr + 8 * (s >> 1) : xr;
        c = ((two ? s & 1 : s) * 64 * wpr + xl) * 8;
        return row < p.M && c < p.K;
    };
    if constexpr (FUSED) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            int row, c;
            if (x_at(s, row, c)) load8((const E*)p.x + row * p.ldx, c, p.K, xv[s]);
        }
    }
    const int8_t* wp[NT];
    const int8_t* ap[MT];
#pragma unroll
    for (int j = 0; j < NT; ++j) wp[j] = p.W + (int64_t)min(n0 + j * 16 + l16, p.N - 1) * p.ldw;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int m = min(i * 16 + l16, p.M - 1);
        ap[i] = FUSED ? xq + m * ldq : p.A + (int64_t)m * p.lda;
    }
    i4 w[2][UK][NT], a[2][FUSED ? 1 : UK][MT];
    auto load = [&](int kb, int set) __attribute__((always_inline)) {   // UK pieces from kb on
        if (kb + UK * 512 <= p.K) {
#pragma unroll
            for (int u = 0; u < UK; ++u) {
#pragma unroll
                for (int j = 0; j < NT; ++j) w[set][u][j] = *(const i4u*)(wp[j] + kb + u * 512 + k0);
                if constexpr (!FUSED) {
#pragma unroll
                    for (int i = 0; i < MT; ++i) a[set][u][i] = *(const i4u*)(ap[i] + kb + u * 512 + k0);
                }
            }
        } else {
#pragma unroll
            for (int u = 0; u < UK; ++u) {
                const int k = kb + u * 512 + k0;
                if (kb + u * 512 >= p.K) {
#pragma unroll
                    for (int j = 0; j < NT; ++j) w[set][u][j] = i4{};
                    if constexpr (!FUSED) {
#pragma unroll
                        for (int i = 0; i < MT; ++i) a[set][u][i] = i4{};
                    }
                    continue;
                }
#pragma unroll
                for (int j = 0; j < NT; ++j) w[set][u][j] = load16(wp[j], k, p.K);
                if constexpr (!FUSED) {
#pragma unroll
                    for (int i = 0; i < MT; ++i) a[set][u][i] = load16(ap[i], k, p.K);
                }
            }
        }
    };
    load(0, 0);
    if constexpr (FUSED) {
        uint32_t* wm = (uint32_t*)red;                     // [2][8] the waves' magnitudes
        uint32_t mx[2] = {0, 0};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            int row, c;
            if (x_at(s, row, c)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    uint32_t& m = mx[s >> 1];
                    m = max(m, mag(xv[s][i]));
                }
            }
        }
        if (!two) mx[0] = max(mx[0], mx[1]);
#pragma unroll
        for (int o = 32; o; o >>= 1) {
            mx[0] = max(mx[0], (uint32_t)__shfl_xor((int)mx[0], o));
            mx[1] = max(mx[1], (uint32_t)__shfl_xor((int)mx[1], o));
        }
        if (lane == 0) {
            wm[wave] = mx[0];
            wm[8 + wave] = mx[1];
        }
        __syncthreads();
        float sc[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t m = 0;
            for (int i = 0; i < wpr; ++i) m = max(m, wm[8 * h + xr * wpr + i]);
            sc[h] = scale_of(m);
        }
        if (xl == 0 && xr < p.M) sa_l[xr] = sc[0];
        if (two && xl == 0 && xr + 8 < p.M) sa_l[xr + 8] = sc[1];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            int row, c;
            if (x_at(s, row, c)) {
                const float f = two ? sc[s >> 1] : sc[0];
                const bool zero = !(f > 0.f);
                *(uint2*)(xq + row * ldq + c) = make_uint2(zero ? 0u : quant4(xv[s], f), zero ? 0u : quant4(xv[s] + 4, f));
            }
        }
        __syncthreads();
    }
    i4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = i4{};
    auto compute = [&](int kb, int set) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < UK; ++u)
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                i4 av;
                if constexpr (FUSED) {
                    // (what stands past K meets zeros of W)
                    const int k = kb + u * 512 + k0;
                    av = *(const i4*)(ap[i] + (k < p.K ? k : 0));
                } else {
                    av = a[set][u][i];
                }
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[set][u][j], av, acc[i][j], 0, 0, 0);
            }
    };
    // the next pieces are on their way while these are multiplied
    constexpr int STEP = UK * 512;
    for (int kb = 0; kb < p.K; kb += 2 * STEP) {
        if (kb + STEP < p.K) load(kb + STEP, 1);
        compute(kb, 0);
        if (kb + STEP < p.K) {
            if (kb + 2 * STEP < p.K) load(kb + 2 * STEP, 0);
            compute(kb + STEP, 1);
        }
    }
    if constexpr (FUSED) __syncthreads();                  // the magnitudes have been read
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) red[((wave * MT + i) * NT + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    // lane: token l16 of a tile, W's rows 4 kg .. 4 kg + 3
    for (int e = tid; e < MT * NT * 64; e += 512) {
        i4 t{};
#pragma unroll
        for (int k = 0; k < 8; ++k) t += red[k * MT * NT * 64 + e];
        const int j = (e >> 6) % NT, i = (e >> 6) / NT, m = i * 16 + (e & 15), n = n0 + j * 16 + 4 * ((e >> 4) & 3);
        if (m >= p.M) continue;
        const float sa = FUSED ? sa_l[m] : p.sa[m];
        E* y = (E*)p.Y + (int64_t)m * p.N + n;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (n + r < p.N) put(y + r, scaled(t[r], sa, p.sw[n + r], p.bias ? p.bias[n + r] : 0.f));
    }
}

// ===========================================================================
// Builders
// ===========================================================================
void build_quant_i8(const QuantI8Params& p0, LaunchRec* rec) {
    // a wave a row up to 2048 columns (its 32 elements a lane), else the
    // workgroup (bf16, a wave / a workgroup, us: 8192 x 1024 8.1 / 11.7, 8192 x
    // 2048 15.5 / 15.9, 8192 x 4096 29.0 / 23.7)
    const bool wave_row = p0.ldq <= 2048;
    QuantI8Params p = p0;
    p.row_blocks = (int32_t)(wave_row ? (p.rows + 3) / 4 : p.rows);
    const int64_t copy = std::min<int64_t>((p.wrows * (p.ldq / 16) + 1023) / 1024, 4096);   // four vectors a thread
    rec->grid = dim3((unsigned)(p.row_blocks + copy), 1, 1);
    rec->block = dim3(256, 1, 1);
    rec->name = "quant_rows_i8";
#define QX_K(E) rec->fn = wave_row ? (const void*)k_quant_i8<E, 1> : (const void*)k_quant_i8<E, 4>;
    if (p.type == FT_F32) { QX_K(float) }
    else if (p.type == FT_F16) { QX_K(Half) }
    else { QX_K(Bf16) }
#undef QX_K
    rec->set_params(p);
}

// Few rows go to the kernel that is made for them, whose waves share K (these /
// 64 x 64 tiles, us: 17 x 256 x 256 3.6 / 3.8, 24 x 1024 x 1024 4.3 / 5.9, 24 x
// 1024 x 8192 12.2 / 22.7, 32 x 64 x 16384 23.5 / 41.2, 32 x 4096 x 4096 8.8 /
// 14.0; 48 x 8192 x 4096 21.5 / 15.5, 64 x 8192 x 4096 25.3 / 15.7).
bool rows_i8s(int64_t M) { return M <= 32; }

// Whether the product quantises its activations itself (x, no A).  Its threads
// are shared among the next power of two of rows, each of whose threads hold
// 32 elements: 16384 columns for one row, 4096 for three, 1024 for nine.
bool fused_i8s(int64_t M, int64_t K) {
    int64_t rows = 1;
    while (rows < M) rows *= 2;
    return rows <= kFusedRows && rows * K <= kFusedElems;
}

void build_gemm_i8s(const GemmI8sParams& p0, bool aligned, LaunchRec* rec, int* tile_m, int* tile_n, int* tile_k) {
    GemmI8sParams p = p0;
    *tile_k = 128;
    if (rows_i8s(p.M)) {
        const bool fused = p.lda == 0;   // no A: x
        // 32 rows of W a workgroup, which halves the reads of A, once there
        // is one for every CU (4096 k, 16 / 32 rows, us: 24 x 8192 16.0 / 12.9,
        // 16 x 8192 13.0 / 11.9, 1 x 8192 10.4 / 11.0, 24 x 4096 9.1 / 11.3)
        const int mt = p.M <= 16 ? 1 : 2, nt = !fused && p.M > 8 && p.N >= 8192 ? 2 : 1;
        *tile_m = 16 * mt;
        *tile_n = 16 * nt;
        rec->grid = dim3((unsigned)((p.N + 16 * nt - 1) / (16 * nt)), 1, 1);
        rec->block = dim3(512, 1, 1);
        rec->shmem = 8 * mt * nt * 1024 + (fused ? 64 + p.M * ((p.K + 15) / 16 * 16 + 16) : 0);
        rec->name = fused ? "linear_i8_rows" : "gemm_i8s_rows";
#define QX_K(E)                                                                    \
    rec->fn = fused ? (const void*)k_skinny_i8s<E, 1, 1, true>                                                       \
            : mt == 1 ? nt == 1 ? (const void*)k_skinny_i8s<E, 1, 1, false> : (const void*)k_skinny_i8s<E, 1, 2, false> \
            : nt == 1 ? (const void*)k_skinny_i8s<E, 2, 1, false> : (const void*)k_skinny_i8s<E, 2, 2, false>;
        if (p.type == FT_F32) { QX_K(float) }
        else if (p.type == FT_F16) { QX_K(Half) }
        else { QX_K(Bf16) }
#undef QX_K
        rec->set_params(p);
        return;
    }
    // The tile whose rounds over the chip take the least: a round's time is
    // close to a start and an end plus so much for each 128 bytes of K, both
    // larger for larger tiles, of which a CU holds one (of the smallest two).
    // us at 64 x 64, 128 x 128, 128 x 256, 256 x 256:
    //   1024 x 1024 x 4096   15   30   41   65       2560 x 4096 x 4096   92   87   85   69
    //   2048 x 2048 x 4096   37   32   43   67       4096 x 2048 x 1024   29   31   23   35
    //   2304 x 2304 x 4096   50   58   43   68       100 x 65536 x 1024   29   33   23   32
    //   8192 x 8192 x 256   131  171  103  101       200 x 8192 x 4096    19   29   41   65
    static const struct { int bm, bn, slots; double ends, step; } kTiles[] = {
        {64, 64, 512, 3.7, 0.45}, {128, 128, 256, 10, 0.66}, {128, 256, 256, 12, 0.94}, {256, 256, 256, 22, 1.45}};
    int bm = 0, bn = 0;
    double least = 0;
    for (const auto& c : kTiles) {
        const int64_t tiles = ((int64_t)(p.M + c.bm - 1) / c.bm) * ((p.N + c.bn - 1) / c.bn);
        const double t = (double)((tiles + c.slots - 1) / c.slots) * (c.ends + c.step * ((p.K + 127) / 128));
        if (bm == 0 || t < least) bm = c.bm, bn = c.bn, least = t;
    }
    const bool al = aligned && p.ldw % 16 == 0 && p.lda % 16 == 0;
    p.tiles_m = (p.M + bm - 1) / bm;
    p.tiles_n = (p.N + bn - 1) / bn;
    const int t = bm + bn;
    rec->grid = dim3((unsigned)((int64_t)p.tiles_m * p.tiles_n), 1, 1);
    rec->block = dim3(t >= 384 ? 512 : 256, 1, 1);
    rec->name = t == 512 ? "gemm_i8s_256x256" : t == 384 ? "gemm_i8s_128x256" : t == 256 ? "gemm_i8s_128x128" : "gemm_i8s_64x64";
#define QX_K(E, A)                                                                     \
    rec->fn = t == 512 ? (const void*)k_gemm_i8s<E, 256, 256, 2, 4, 2, A>              \
            : t == 384 ? (const void*)k_gemm_i8s<E, 128, 256, 2, 4, A ? 3 : 2, A>      \
            : t == 256 ? (const void*)k_gemm_i8s<E, 128, 128, 2, 2, A ? 4 : 2, A>      \
                       : (const void*)k_gemm_i8s<E, 64, 64, 2, 2, A ? 4 : 2, A>;
#define QX_A(E) if (al) { QX_K(E, true) } else { QX_K(E, false) }
    if (p.type == FT_F32) { QX_A(float) }
    else if (p.type == FT_F16) { QX_A(Half) }
    else { QX_A(Bf16) }
#undef QX_A
#undef QX_K
    *tile_m = bm;
    *tile_n = bn;
    rec->set_params(p);
}

}  // namespace qx
