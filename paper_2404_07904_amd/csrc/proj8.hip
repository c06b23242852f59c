// Matrix product of operands in 8-bit floating point with power-of-two scales for blocks of 128 along the contraction:
//
//     C[m][n] = act(bias[n] + sum_b 2^(sa[m][b] + sb[n][b]) sum_{k in block b} a[m][k] b[n][k])
//
// Both operands lie with the contraction index contiguous, as hgrn2_quant8 writes them; a training step's three products
// (x W^T, dY W, dY^T x) are this one with operands taken from one or the other order.  The scaled matrix instructions of gfx950 apply the scales
// themselves, so a sum runs through the whole contraction in its fp32 accumulators; they are 2^(byte - 127) per row and block of 32, and all
// four blocks of a block of 128 get the same byte.  (Which 32 of the 128 values of a step a lane holds does not matter then, as long as
// both operands have the same ones.)
// Precision: these instructions (and the unscaled ones in 8 bits alike) add the products eight by eight and cut off what lies 2^-13 below the largest of the
// eight, 1.5e-5 of a sum of random terms at any length; from there on sums are fp32.  Results in bf16, whose own rounding is up to 2^-8, are such sums, with the
// same eights in every kernel: one token's result and the same token's among many differ by the order of fp32 additions only.  Results in fp32 are exact sums: a
// value of e4m3 times its scale is a value of bf16, so their fragments are converted on the way from LDS to the bf16 instructions, which add
// products in fp32 (4e-8 at K = 1024, as fp32 additions one after the other).
//
// Bound by the matrix units where rows are many: 16384 x 2048 x 8192 (M, N, K) 220 us, 2.5 PFLOP/s, the steady state of the steps; with K = 2048
// the start and end of a tile, which are not overlapped with another's, bring 16384 x 8192 to 2.1 PFLOP/s (260 us).  Four waves of 128 x 128 instead of
// eight of 128 x 64: 226 us for 220.  Exact sums: bound by the conversions, 16 cycles for two values a lane, of which a wave of 128 x 128 needs the fewest next to
// its products: 2048 x 8192 x 16384 385 us, 1.43 PFLOP/s (tiles of 128 x 128 546; in bf16 217).  Hundreds of rows: bound by the time of few steps on part of the
// units.  Few rows: by reading B (1 x 8192 x 2048 4.7 to 5.0 us for either type).
#include <type_traits>

#include "../../include/hgrn2.h"
#include "common.hpp"
#include "mixer.hpp"
#include "proj8_plan.hpp"

namespace hgrn2 {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// Exact sums: 32 bytes of a row and their scale become four fragments of the bf16 instructions.  All values are taken at half their size: the largest,
// 2^128, is then a number of bf16 too; sums come out a quarter of theirs.
constexpr float kExactBack = 4.0f;
// (Half of 2^(byte - 127): the conversion goes by the exponent's bits, 0 for 2^-127 and 255 for what is no number.  There is no half of byte 0, which counts as 1.)
__device__ __forceinline__ float exact_scale(int byte)
{
    const int least = max(byte, 1);
    return __uint_as_float((uint32_t)(least - (least < 255 ? 1 : 0)) << 23);
}
__device__ __forceinline__ bf16x8 exact_part(const i32x8& f, int u, float scale)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)f[2 * u], scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)f[2 * u], scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)f[2 * u + 1], scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)f[2 * u + 1], scale, true);
    return __builtin_shufflevector(__builtin_shufflevector(a, b, 0, 1, 2, 3), __builtin_shufflevector(c, d, 0, 1, 2, 3), 0, 1, 2, 3, 4, 5, 6, 7);
}

struct Proj8Params {
    const uint8_t *A, *B, *sa, *sb;
    int M, N, K;              // K: bytes of a row, a multiple of 128
    int sp;                   // bytes of a row of scales
    int ra, rb;               // log2 of the rows that share a scale: 0 or 7
    const float* bias;
    int act;                  // hgrn2_act
    void* C;
    float* shares;            // [split][M][N], where the contraction is split
    int splits;
};

template <int ACT> __device__ __forceinline__ float proj8_act(float v)
{
    return ACT == HGRN2_ACT_SILU ? mixer_silu(v) : ACT == HGRN2_ACT_SIGMOID ? mixer_sigmoid(v) : v;
}
__device__ __forceinline__ float proj8_act(int act, float v)
{
    return act == HGRN2_ACT_SILU ? mixer_silu(v) : act == HGRN2_ACT_SIGMOID ? mixer_sigmoid(v) : v;
}

// Eight numbers to a place that needs no alignment beyond their own.
typedef uint32_t words_of_bf16 __attribute__((ext_vector_type(4), aligned(2)));
typedef float four_floats __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void store_eight(__bf16* to, const float (&v)[8])
{
    words_of_bf16 u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        bf16x2 h;
        h.x = (__bf16)v[2 * e];
        h.y = (__bf16)v[2 * e + 1];
        u[e] = __builtin_bit_cast(uint32_t, h);
    }
    *reinterpret_cast<words_of_bf16*>(to) = u;
}
__device__ __forceinline__ void store_eight(float* to, const float (&v)[8])
{
    *reinterpret_cast<four_floats*>(to) = four_floats{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<four_floats*>(to + 4) = four_floats{v[4], v[5], v[6], v[7]};
}

// Places for four steps' scales: those in use and those on their way.
constexpr int scale_places(int ns) { return ns <= 4 ? 2 : 4; }

// ---- tiles -----------------------------------------------------------------------------------------------------------
// A workgroup computes a TM x TN tile, WM x WN waves side by side, in steps of 128 along the contraction: whole lines of every row.  NS steps
// lie in LDS; `global_load_lds` fills them, 16 bytes per lane, no registers in between.  Such a load writes the 64 lanes' vectors
// to consecutive addresses, so a row is 128 bytes with no padding, and the 16-byte piece c of row r is kept at position
// c ^ ((r >> 1) & 7): 16 consecutive rows then cover all 64 banks for any piece.  One barrier a step, before its second half: by then every
// wave has that half's fragments in registers and the next step's loads, which went out NS - 1 steps ago, have landed; behind it the step's
// place is refilled with the step NS later.  Scales come four steps at a time, a dword per row, the same way.
template <typename OUT, int TM, int TN, int WM, int WN, int NS>
__global__ __launch_bounds__(64 * WM * WN, TM * TN / (WM * WN) > 8192 ? 1 : 2) void proj8_tile_kernel(Proj8Params p)
{
    constexpr int NW = WM * WN, LA = TM / 8 / NW, LB = TN / 8 / NW, NI = TM / WM / 32, NJ = TN / WN / 32;
    constexpr int STEP = (TM + TN) * 128, SCALES = NS * STEP, ROWS = TM + TN, LS = (ROWS / 64 + NW - 1) / NW;
    constexpr bool EXACT = sizeof(OUT) == 4;
    static_assert((NS & (NS - 1)) == 0 && NS >= 2 && NS <= 8, "places of a power of two");
    static_assert(LA >= 1 && LB >= 1 && NI >= 1 && NJ >= 1 && ROWS % 64 == 0, "whole load instructions");
    static_assert((NS - 1) * (LA + LB + LS) < 64, "loads that can be counted");
    typedef __attribute__((address_space(3))) void* lds_ptr;
    typedef const __attribute__((address_space(1))) void* global_ptr;
    extern __shared__ __align__(16) char smem[];
    const int tid = (int)threadIdx.x, lane = tid & 63, r32 = lane & 31, g = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w / WN, wn = w % WN;
    // tiles of an XCD lie together, in bands of a few rows of tiles
    const int n_bm = (p.M + TM - 1) / TM, n_bn = (p.N + TN - 1) / TN;
    int m0, n0;
    {
        const int tiles = n_bm * n_bn, id = (int)blockIdx.x, per = tiles / 8, rem = tiles - per * 8, x = id % 8;
        const int t = x * per + min(x, rem) + id / 8;
        constexpr int BAND = 4;
        const int band = t / (BAND * n_bn), in = t - band * BAND * n_bn, rows = min(BAND, n_bm - band * BAND);
        m0 = (band * BAND + in % rows) * TM;
        n0 = in / rows * TN;
    }
    const int steps = p.K / 128, groups = (steps + 3) / 4;
    const int first = (int)((long long)blockIdx.y * groups / p.splits) * 4;
    const int nk = min((int)((long long)(blockIdx.y + 1) * groups / p.splits) * 4, steps) - first;
    // rows past an operand's end re-read its last one
    uint32_t ao[LA], bo[LB];
    const char* abase = reinterpret_cast<const char*>(p.A) + (size_t)m0 * p.K + (size_t)first * 128;
    const char* bbase = reinterpret_cast<const char*>(p.B) + (size_t)n0 * p.K + (size_t)first * 128;
#pragma unroll
    for (int j = 0; j < LA; ++j) {
        const int row = 8 * (LA * w + j) + (lane >> 3);
        ao[j] = (uint32_t)min(row, p.M - 1 - m0) * (uint32_t)p.K + (((lane & 7) ^ ((row >> 1) & 7)) << 4);
    }
#pragma unroll
    for (int j = 0; j < LB; ++j) {
        const int row = 8 * (LB * w + j) + (lane >> 3);
        bo[j] = (uint32_t)min(row, p.N - 1 - n0) * (uint32_t)p.K + (((lane & 7) ^ ((row >> 1) & 7)) << 4);
    }
    // step ks (its last one again behind the end) into place `at` of the two
    auto load_a = [&](int at, int ks, int j) {
        __builtin_amdgcn_global_load_lds((global_ptr)(abase + (size_t)min(ks, nk - 1) * 128 + ao[j]), (lds_ptr)(smem + at * STEP + 8 * (LA * w + j) * 128), 16, 0, 0);
    };
    auto load_b = [&](int at, int ks, int j) {
        __builtin_amdgcn_global_load_lds((global_ptr)(bbase + (size_t)min(ks, nk - 1) * 128 + bo[j]), (lds_ptr)(smem + at * STEP + TM * 128 + 8 * (LB * w + j) * 128), 16, 0, 0);
    };
    // scales of the tile's rows of A and B, 64 rows a load and four steps of them; LS such loads a wave
    const char* srow[LS];
    int sr[LS];
#pragma unroll
    for (int j = 0; j < LS; ++j) {
        sr[j] = 64 * ((w + j * NW) % (ROWS / 64));
        const int row = sr[j] < TM ? min(m0 + sr[j] + lane, p.M - 1) >> p.ra : min(n0 + sr[j] - TM + lane, p.N - 1) >> p.rb;
        srow[j] = reinterpret_cast<const char*>(sr[j] < TM ? p.sa : p.sb) + (size_t)row * p.sp + first;
    }
    auto load_scales = [&](int ks) {
#pragma unroll
        for (int j = 0; j < LS; ++j)
            __builtin_amdgcn_global_load_lds((global_ptr)(srow[j] + (min(ks, nk - 1) & ~3)), (lds_ptr)(smem + SCALES + ((ks >> 2) & (scale_places(NS) - 1)) * ROWS * 4 + sr[j] * 4), 4, 0, 0);
    };
    f32x16 acc[NI][NJ];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    // Fragments of half a step: B's of this half and the next, A's of either: a row of the wave's tile is multiplied and its fragment
    // requested anew for the next half at once.
    i32x8 fa[NI], fb[2][NJ];
    const int sw = (r32 >> 1) & 7;
    auto frag = [&](const char* row, int kk) {
        const i32x4 lo = *reinterpret_cast<const i32x4*>(row + (((4 * kk + 2 * g) ^ sw) << 4));
        const i32x4 hi = *reinterpret_cast<const i32x4*>(row + (((4 * kk + 2 * g + 1) ^ sw) << 4));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto read_a = [&](int at, int kk, int i) { fa[i] = frag(smem + at * STEP + ((TM / WM) * wm + 32 * i + r32) * 128, kk); };
    auto read_b = [&](int at, int kk) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) fb[kk][j] = frag(smem + at * STEP + TM * 128 + ((TN / WN) * wn + 32 * j + r32) * 128, kk);
    };
    int sa[NI], sb[NJ];
    auto read_scales = [&](int ks) {
        const uint8_t* s = reinterpret_cast<const uint8_t*>(smem) + SCALES + ((ks >> 2) & (scale_places(NS) - 1)) * ROWS * 4 + (ks & 3);
#pragma unroll
        for (int i = 0; i < NI; ++i) sa[i] = s[((TM / WM) * wm + 32 * i + r32) * 4];
#pragma unroll
        for (int j = 0; j < NJ; ++j) sb[j] = s[(TM + (TN / WN) * wn + 32 * j + r32) * 4];
    };
    constexpr int NL = LA + LB;
    bf16x8 wb[EXACT ? NJ : 1][4];
    auto multiply = [&](int kk, int i) {
        if constexpr (EXACT) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const bf16x8 wa = exact_part(fa[i], u, exact_scale(sa[i]));
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    if (i == 0) wb[j][u] = exact_part(fb[kk][j], u, exact_scale(sb[j]));
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb[j][u], wa, acc[i][j], 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < NJ; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[kk][j], fa[i], acc[i][j], 0, 0, 0, sb[j], 0, sa[i]);
        }
    };
    auto refill = [&](int at, int ks, int j) { if (j < LB) load_b(at, ks, j); else load_a(at, ks, j - LB); };
#pragma unroll
    for (int k = 0; k < NS; ++k) {
        load_scales(k);
#pragma unroll
        for (int j = 0; j < NL; ++j) refill(k, k, j);
    }
    // all but the youngest n of this wave's loads have landed, and all its LDS reads
    constexpr auto landed = [](int n) { return (n & 15) | ((n >> 4) << 14) | 0x0070; };
    __builtin_amdgcn_s_waitcnt(landed((NS - 1) * (NL + LS)));
    __builtin_amdgcn_s_barrier();
    read_scales(0);
    read_b(0, 0);
#pragma unroll
    for (int i = 0; i < NI; ++i) read_a(0, 0, i);
    // (No branch inside a step: the compiler would move the multiplications past it.  The last steps request and read once more what
    // nobody uses.)
    for (int k = 0; k < nk; ++k) {
        const int at = k & (NS - 1), behind = (k + 1) & (NS - 1);
        __builtin_amdgcn_sched_barrier(0);
        multiply(0, 0);
        __builtin_amdgcn_sched_barrier(0);
        read_b(at, 1);
        read_a(at, 1, 0);
#pragma unroll
        for (int i = 1; i < NI; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            multiply(0, i);
            __builtin_amdgcn_sched_barrier(0);
            read_a(at, 1, i);
        }
        __builtin_amdgcn_sched_barrier(0);
        multiply(1, 0);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(landed((NS - 2) * (NL + LS)));           // this wave's loads of the next step, its fragments of this one
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        read_b(behind, 0);
        read_a(behind, 0, 0);
        load_scales(k + NS);
#pragma unroll
        for (int i = 1; i < NI; ++i) {
#pragma unroll
            for (int j = 0; j < NL; ++j)
                if (j * (NI - 1) / NL == i - 1) refill(at, k + NS, j);
            __builtin_amdgcn_sched_barrier(0);
            multiply(1, i);
            __builtin_amdgcn_sched_barrier(0);
            read_a(behind, 0, i);
        }
        if constexpr (NI == 1) {
#pragma unroll
            for (int j = 0; j < NL; ++j) refill(at, k + NS, j);
        }
        read_scales(k + 1);
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    // acc[i][j][v] = C[m0 + (TM / WM) wm + 32 i + r32][n0 + (TN / WN) wn + 32 j + 8 (v / 4) + 4 g + v % 4]; a wave's rows leave through a
    // place of its own in LDS, 32 x 32 NJ at a time, as whole pieces of rows: eight columns a lane, the same ones for all its rows
    constexpr int PITCH = 32 * NJ + 4, PER = NJ * 32 / 8;           // floats of a row; lanes of a row
    float* stage = reinterpret_cast<float*>(smem) + w * 32 * PITCH;
    static_assert(NW * 32 * PITCH * 4 <= NS * STEP, "the stages fit where the steps were");
    const int c = (lane % PER) * 8, n = n0 + (TN / WN) * wn + c, mw = m0 + (TM / WM) * wm + lane / PER;
    float bias[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = 0.0f;
    if (p.bias && p.splits == 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) bias[e] = p.bias[min(n + e, p.N - 1)];
    }
    auto leave = [&](auto ACT, auto WHOLE, auto* out) {
        typedef std::remove_pointer_t<decltype(out)> T;
        constexpr bool whole = decltype(WHOLE)::value;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<f32x4*>(stage + r32 * PITCH + 32 * j + 8 * q + 4 * g) = f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int k = 0; k < 32 * PER / 64; ++k) {
                const int r = k * (64 / PER), m = mw + 32 * i + r;
                const f32x4 lo = *reinterpret_cast<const f32x4*>(stage + (r + lane / PER) * PITCH + c), hi = *reinterpret_cast<const f32x4*>(stage + (r + lane / PER) * PITCH + c + 4);
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = proj8_act<decltype(ACT)::value>((EXACT ? kExactBack : 1.0f) * (e < 4 ? lo[e & 3] : hi[e & 3]) + bias[e]);
                T* to = out + (size_t)m * p.N + n;
                if (whole || m < p.M) {
                    if (whole || n + 8 <= p.N) store_eight(to, v);
                    else
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (n + e < p.N) to[e] = (T)v[e];
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    };
    const bool whole = m0 + TM <= p.M && n0 + TN <= p.N;
    auto as = [&](auto ACT, auto* out) {
        if (whole) leave(ACT, std::true_type(), out);
        else leave(ACT, std::false_type(), out);
    };
    float* share = p.shares + (size_t)blockIdx.y * p.M * p.N;
    typedef std::integral_constant<int, HGRN2_ACT_NONE> None;
    if constexpr (sizeof(OUT) == 2) {
        if (p.splits > 1) { as(None(), share); return; }
    }
    // (each of these once: what is written out twice is not inlined, and its sums pass through memory)
    OUT* out = sizeof(OUT) == 4 && p.splits > 1 ? reinterpret_cast<OUT*>(share) : static_cast<OUT*>(p.C);
    const int act = p.splits > 1 ? HGRN2_ACT_NONE : p.act;
    if (act == HGRN2_ACT_SILU) as(std::integral_constant<int, HGRN2_ACT_SILU>(), out);
    else if (act == HGRN2_ACT_SIGMOID) as(std::integral_constant<int, HGRN2_ACT_SIGMOID>(), out);
    else as(None(), out);
}

// The shares of a split contraction added up in order, bias and activation.
template <typename OUT>
__global__ __launch_bounds__(kThreads) void proj8_sums_kernel(Proj8Params p)
{
    const size_t n = (size_t)p.M * p.N, e = ((size_t)blockIdx.x * kThreads + threadIdx.x) * 4;
    if (e >= n) return;
    const int left = (int)min(n - e, (size_t)4);
    float v[4], s[4];
    load_row<float, 4>(p.shares + e, left, v);
    for (int k = 1; k < p.splits; ++k) {
        load_row<float, 4>(p.shares + (size_t)k * n + e, left, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += s[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) v[i] = proj8_act(p.act, v[i] + (p.bias ? p.bias[(e + i) % p.N] : 0.0f));
    store_row<OUT, 4>(static_cast<OUT*>(p.C) + e, left, v);
}

// ---- few rows ---------------------------------------------------------------------------------------------------------
// Up to 16 MI rows of A (tokens): bound by reading B once.  A workgroup takes 16 rows of B; its waves take every eighth block of the
// contraction each, straight from memory to the matrix instructions (a lane's 32 bytes of a row lie next to its neighbours'), and
// add up in LDS.
template <typename OUT, int MI>
__global__ __launch_bounds__(512) void proj8_rows_kernel(Proj8Params p)
{
    constexpr int W = 8;
    constexpr bool EXACT = sizeof(OUT) == 4;
    __shared__ __align__(16) f32x4 red[W][MI][64];
    const int tid = (int)threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n0 = (int)blockIdx.x * 16, steps = p.K / 128;
    const int nr = min(n0 + r, p.N - 1);
    const uint8_t* b = p.B + (size_t)nr * p.K + 32 * g;
    const uint8_t* sb = p.sb + (size_t)(nr >> p.rb) * p.sp;
    const uint8_t *a[MI], *sa[MI];
    f32x4 acc[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        const int mr = min(16 * i + r, p.M - 1);
        a[i] = p.A + (size_t)mr * p.K + 32 * g;
        sa[i] = p.sa + (size_t)(mr >> p.ra) * p.sp;
        acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    auto vec = [](const uint8_t* q) {
        const i32x4 lo = *reinterpret_cast<const i32x4*>(q), hi = *reinterpret_cast<const i32x4*>(q + 16);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    for (int k = w; k < steps; k += W) {
        const i32x8 fb = vec(b + (size_t)k * 128);
        const int eb = sb[k];
#pragma unroll
        for (int i = 0; i < MI; ++i)
            if constexpr (EXACT) {
                const i32x8 fa = vec(a[i] + (size_t)k * 128);
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(exact_part(fb, u, exact_scale(eb)), exact_part(fa, u, exact_scale(sa[i][k])), acc[i], 0, 0, 0);
            } else {
                acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb, vec(a[i] + (size_t)k * 128), acc[i], 0, 0, 0, eb, 0, (int)sa[i][k]);
            }
    }
#pragma unroll
    for (int i = 0; i < MI; ++i) red[w][i][lane] = acc[i];
    __syncthreads();
    // acc[i][v] = C[16 i + r][n0 + 4 g + v]
    for (int i = w; i < MI; i += W) {
        f32x4 s = red[0][i][lane];
#pragma unroll
        for (int k = 1; k < W; ++k) s += red[k][i][lane];
        const int m = 16 * i + r, n = n0 + 4 * g;
        if (m < p.M && n < p.N) {
            const int left = p.N - n;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = proj8_act(p.act, (EXACT ? kExactBack : 1.0f) * s[e] + (p.bias ? p.bias[min(n + e, p.N - 1)] : 0.0f));
            store_row<OUT, 4>(static_cast<OUT*>(p.C) + (size_t)m * p.N + n, left, v);
        }
    }
}

namespace {

template <typename OUT, int TM, int TN, int WM, int WN, int NS> hipError_t launch_tile(const Proj8Params& p, hipStream_t st)
{
    constexpr int LDS = NS * (TM + TN) * 128 + scale_places(NS) * (TM + TN) * 4;
    static_assert(LDS <= 160 * 1024, "the tiles fit");
    const void* k = reinterpret_cast<const void*>(&proj8_tile_kernel<OUT, TM, TN, WM, WN, NS>);
    const hipError_t e = allow_dynamic_lds(k, LDS);
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)(((p.M + TM - 1) / TM) * ((p.N + TN - 1) / TN)), (unsigned)p.splits);
    proj8_tile_kernel<OUT, TM, TN, WM, WN, NS><<<grid, 64 * WM * WN, LDS, st>>>(p);
    return hipGetLastError();
}

template <typename OUT> hipError_t launch_proj8(const Proj8Params& p, const Proj8Plan& plan, hipStream_t st)
{
    if (plan.tile == 0) {
        const dim3 grid((unsigned)((p.N + 15) / 16));
        if (p.M <= 16) proj8_rows_kernel<OUT, 1><<<grid, 512, 0, st>>>(p);
        else if (p.M <= 32) proj8_rows_kernel<OUT, 2><<<grid, 512, 0, st>>>(p);
        else proj8_rows_kernel<OUT, 4><<<grid, 512, 0, st>>>(p);
        return hipGetLastError();
    }
    hipError_t e;
    if (plan.tile == 64) e = launch_tile<OUT, 64, 64, 2, 2, 8>(p, st);
    else if (plan.tile == 128) e = launch_tile<OUT, 128, 128, 2, 2, 4>(p, st);
    else e = launch_tile<OUT, 256, 256, 2, sizeof(OUT) == 4 ? 2 : 4, 2>(p, st);
    if (e != hipSuccess || p.splits == 1) return e;
    proj8_sums_kernel<OUT><<<dim3((unsigned)(((size_t)p.M * p.N + 4 * kThreads - 1) / (4 * kThreads))), kThreads, 0, st>>>(p);
    return hipGetLastError();
}

int proj8_check(int M, int N, int K, int out_dtype)
{
    if (M < 0 || N < 0 || K <= 0 || K > 0x7fffff00 || (out_dtype != HGRN2_F32 && out_dtype != HGRN2_BF16)) return HGRN2_ERR_SHAPE;
    if (M > 0x7ffffe00 || N > 0x7ffffe00) return HGRN2_ERR_SHAPE;
    // a tile's rows are found with 32-bit offsets
    if (hgrn2_quant8_pitch(K) > (1 << 23)) return HGRN2_ERR_UNSUPPORTED;
    if ((((long long)M + 63) / 64) * (((long long)N + 63) / 64) > 0x7fffffffll) return HGRN2_ERR_UNSUPPORTED;
    return HGRN2_OK;
}

}   // namespace

}   // namespace hgrn2

using namespace hgrn2;

extern "C" {

size_t hgrn2_proj8_workspace_bytes(int32_t M, int32_t N, int32_t K)
{
    if (proj8_check(M, N, K, HGRN2_BF16) != HGRN2_OK || M == 0 || N == 0) return 0;
    // (of either type of results)
    const int steps = hgrn2_quant8_pitch(K) / 128, a = plan_proj8(M, N, steps).splits, b = plan_proj8(M, N, steps, true).splits, splits = a > b ? a : b;
    return splits > 1 ? ((size_t)splits * M * N * 4 + 255) & ~(size_t)255 : 0;
}

int hgrn2_proj8(int32_t M, int32_t N, int32_t K, const uint8_t* a, const uint8_t* a_scale, int32_t a_rows, const uint8_t* b, const uint8_t* b_scale,
                int32_t b_rows, const float* bias, int32_t act, int32_t out_dtype, void* c, void* ws, size_t ws_bytes, void* stream)
{
    const int rc = proj8_check(M, N, K, out_dtype);
    if (rc != HGRN2_OK) return rc;
    if (act < HGRN2_ACT_NONE || act > HGRN2_ACT_SIGMOID) return HGRN2_ERR_SHAPE;
    if ((a_rows != 1 && a_rows != 128) || (b_rows != 1 && b_rows != 128)) return HGRN2_ERR_UNSUPPORTED;
    if (M == 0 || N == 0) return HGRN2_OK;
    if (!a || !a_scale || !b || !b_scale || !c) return HGRN2_ERR_NULL;
    if ((((uintptr_t)a | (uintptr_t)b) & 15) || (((uintptr_t)a_scale | (uintptr_t)b_scale) & 3)) return HGRN2_ERR_UNSUPPORTED;
    const int pitch = hgrn2_quant8_pitch(K);
    const Proj8Plan plan = plan_proj8(M, N, pitch / 128, out_dtype == HGRN2_F32);
    const long long tile = plan.tile, groups = tile ? ((M + tile - 1) / tile) * ((N + tile - 1) / tile) : ((long long)N + 15) / 16;
    if (!launchable(groups, tile == 0 || (tile == 256 && out_dtype == HGRN2_BF16) ? 512 : 256)) return HGRN2_ERR_UNSUPPORTED;
    if (plan.splits > 1 && (!ws || ws_bytes < hgrn2_proj8_workspace_bytes(M, N, K) || ((uintptr_t)ws & 255))) return HGRN2_ERR_WORKSPACE;
    Proj8Params p{a, b, a_scale, b_scale, M, N, pitch, hgrn2_quant8_scale_pitch(K), a_rows == 128 ? 7 : 0, b_rows == 128 ? 7 : 0, bias, act, c,
                  static_cast<float*>(ws), plan.splits};
    hipStream_t st = static_cast<hipStream_t>(stream);
    const hipError_t e = out_dtype == HGRN2_BF16 ? launch_proj8<__bf16>(p, plan, st) : launch_proj8<float>(p, plan, st);
    return e == hipSuccess ? HGRN2_OK : HGRN2_ERR_HIP;
}

}   // extern "C"
