// Quantisation to 8-bit floating point (e4m3: 4 exponent, 3 mantissa bits, largest value 448) with a power-of-two scale for each
// block of 128 along a row (and of 1 or 128 rows):
//
//     scale = 2^e, the smallest with max |x| <= 448 * 2^e over the block;     q = e4m3(x / scale), ties to even
//
// A power of two costs a floating-point format at most the one bit of its smallest values, dividing by it is exact, and the matrix
// instructions of gfx950 apply such scales themselves (proj8.hip), held as they take them: the byte e + 127.  Blocks whose largest value is
// below 2^-100 take the scale of 2^-100, so that exponents stay in range.
// Values that are not finite do not enter their block's scale and become NaN.
//
// Bound by memory: one workgroup takes 128 x 128 values (or 16 x 128), 16 bytes of bf16 per lane and load, keeps them in
// registers, finds the largest of every row (16 lanes), column or of the whole tile, and writes the tile in one or both orders, each in its
// own scales.  16384 x 8192 in bf16: rows 75 us (5.4 TB/s), both orders 113 us (4.8 TB/s; a copy reaches 4.8).  So it is with values kept as
// they came (two to a register: as floats they spilled, 199 us) and their magnitudes compared as integers.
#include "../../include/hgrn2.h"
#include "common.hpp"
#include "mixer.hpp"

namespace hgrn2 {

struct QuantParams {
    const void* x;
    long long ldx;
    int M, K, pitch, pitch_t;             // pitches of q and qT: K and M rounded up to 128
    int sp, sp_t;                         // bytes of a row of scales: blocks of a row rounded up to 4
    int blocks, blocks_t;                 // blocks of 128 of a row, of a column
    uint8_t *q, *s, *qt, *st;
};

// Byte of the scale for the largest magnitude (bits of a finite float): 448 = 1.75 * 2^8.
__device__ __forceinline__ uint32_t scale_byte(uint32_t most)
{
    most = max(most, 27u << 23);                                     // 2^-100
    return (most >> 23) - 8u + ((most & 0x7fffffu) > 0x600000u ? 1u : 0u);
}
__device__ __forceinline__ float scale_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Eight values of a row as they come, and their magnitudes, which compare as integers: two to a word in bf16.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <typename IO> struct Eight;
template <> struct Eight<__bf16> {
    static constexpr int W = 4;
    typedef u16x2 Mag;
    uint32_t w[W];
    __device__ __forceinline__ float value(int i) const { return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
    __device__ __forceinline__ void set(int i, __bf16 v) { w[i >> 1] |= (uint32_t)__builtin_bit_cast(uint16_t, v) << (16 * (i & 1)); }
    template <bool ODD> __device__ __forceinline__ Mag magnitude(int k) const
    {
        u16x2 m = __builtin_bit_cast(u16x2, w[k] & 0x7fff7fffu);
        if (ODD) {
            if (m[0] >= 0x7f80) m[0] = 0;
            if (m[1] >= 0x7f80) m[1] = 0;
        }
        return m;
    }
    static __device__ __forceinline__ uint32_t bits(Mag m) { return (uint32_t)max(m[0], m[1]) << 16; }                 // the larger one's, as a float's
    static __device__ __forceinline__ uint32_t bits_of(Mag m, int i) { return (uint32_t)m[i & 1] << 16; }
};
template <> struct Eight<float> {
    static constexpr int W = 8;
    typedef uint32_t Mag;
    uint32_t w[W];
    __device__ __forceinline__ float value(int i) const { return __uint_as_float(w[i]); }
    __device__ __forceinline__ void set(int i, float v) { w[i] = __float_as_uint(v); }
    template <bool ODD> __device__ __forceinline__ Mag magnitude(int k) const
    {
        const uint32_t m = w[k] & 0x7fffffffu;
        return ODD && m >= 0x7f800000u ? 0u : m;
    }
    static __device__ __forceinline__ uint32_t bits(Mag m) { return m; }
    static __device__ __forceinline__ uint32_t bits_of(Mag m, int) { return m; }
};
__device__ __forceinline__ u16x2 larger(u16x2 a, u16x2 b) { return __builtin_elementwise_max(a, b); }
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max(a, b); }

template <int CTRL> __device__ __forceinline__ uint32_t dpp_u(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
// the largest over the 16 lanes of a row
__device__ __forceinline__ uint32_t max16(uint32_t v)
{
    v = max(v, dpp_u<0x128>(v));
    v = max(v, dpp_u<0x124>(v));
    v = max(v, dpp_u<0x122>(v));
    return max(v, dpp_u<0x121>(v));
}
// over the four rows of a wave
template <typename T> __device__ __forceinline__ T max_rows(T v)
{
    uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    u = __builtin_bit_cast(uint32_t, larger(__builtin_bit_cast(T, (uint32_t)r[0]), __builtin_bit_cast(T, (uint32_t)r[1])));
    const auto q = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return larger(__builtin_bit_cast(T, (uint32_t)q[0]), __builtin_bit_cast(T, (uint32_t)q[1]));
}
// Four values to bytes.  ODD: an infinity may be among them, which becomes NaN whatever the conversion makes of it.
template <bool ODD> __device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d, float inv)
{
    auto fit = [inv](float v) { return ODD && fabsf(v) == __builtin_inff() ? __uint_as_float(0x7fc00000u) : v * inv; };
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(fit(a), fit(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(fit(c), fit(d), low, true);
}

// J rows of eight columns per lane: tiles of 16 J rows.  BLOCK: a scale for 128 rows; both orders where TR: the second one's bytes are turned
// in LDS, eight rows of a column at a time (piece p of column c at p ^ (c / 8)), and leave as whole lines.
template <typename IO, int J, bool BLOCK, bool TR, bool ODD>
__device__ __forceinline__ void quant8_tile(const QuantParams& p, Eight<IO> (&raw)[J], uint32_t (&col_most)[kWaves][128], uint2 (&turned)[TR ? 128 : 1][16])
{
    typedef Eight<IO> E;
    constexpr int W = E::W, PER = 8 / W;
    const int tid = (int)threadIdx.x, c8 = (tid & 15) * 8, rg = tid >> 4;
    const int kb = (int)blockIdx.x % p.blocks, mb = (int)blockIdx.x / p.blocks, k0 = kb * 128 + c8, m0 = mb * 16 * J + rg * J;
    // from here on the words are what they are: values formed before are formed anew, not kept
    auto forget = [&]() {
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int k = 0; k < W; ++k) asm volatile("" : "+v"(raw[j].w[k]));
    };
    auto largest = [&](int j) {
        typename E::Mag m = raw[j].template magnitude<ODD>(0);
#pragma unroll
        for (int k = 1; k < W; ++k) m = larger(m, raw[j].template magnitude<ODD>(k));
        return E::bits(m);
    };
    uint32_t byte_all = 0;
    if constexpr (BLOCK) {
        uint32_t all = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) all = max(all, largest(j));
        all = max_rows(max16(all));
        if ((tid & 63) == 0) col_most[tid >> 6][0] = all;
        __syncthreads();
        byte_all = scale_byte(max(max(col_most[0][0], col_most[1][0]), max(col_most[2][0], col_most[3][0])));
        if (tid == 0) {
            p.s[(size_t)mb * p.sp + kb] = (uint8_t)byte_all;
            if (TR) p.st[(size_t)kb * p.sp_t + mb] = (uint8_t)byte_all;
        }
    }
    // rows
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const uint32_t byte = BLOCK ? byte_all : scale_byte(max16(largest(j)));
        const float inv = scale_inverse(byte);
        if (m0 + j < p.M) {
            const E& r = raw[j];
            uint2 o;
            o.x = to_e4m3<ODD>(r.value(0), r.value(1), r.value(2), r.value(3), inv);
            o.y = to_e4m3<ODD>(r.value(4), r.value(5), r.value(6), r.value(7), inv);
            *reinterpret_cast<uint2*>(p.q + (size_t)(m0 + j) * p.pitch + k0) = o;
            if (!BLOCK && c8 == 0) p.s[(size_t)(m0 + j) * p.sp + kb] = (uint8_t)byte;
        }
    }
    if constexpr (TR) {
        forget();
        if constexpr (!BLOCK) {
#pragma unroll
            for (int k = 0; k < W; ++k) {
                typename E::Mag m = raw[0].template magnitude<ODD>(k);
#pragma unroll
                for (int j = 1; j < J; ++j) m = larger(m, raw[j].template magnitude<ODD>(k));
                m = max_rows(m);
                if ((tid & 63) < 16)
#pragma unroll
                    for (int i = 0; i < PER; ++i) col_most[tid >> 6][c8 + PER * k + i] = E::bits_of(m, i);
            }
            __syncthreads();
            forget();
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t byte = byte_all;
            if constexpr (!BLOCK) {
                byte = scale_byte(max(max(col_most[0][c8 + i], col_most[1][c8 + i]), max(col_most[2][c8 + i], col_most[3][c8 + i])));
                if (tid < 16 && k0 + i < p.K) p.st[(size_t)(k0 + i) * p.sp_t + mb] = (uint8_t)byte;
            }
            const float inv = scale_inverse(byte);
            auto v = [&](int j) { return raw[j % J].value(i); };
            uint2 o;
            o.x = to_e4m3<ODD>(v(0), v(1), v(2), v(3), inv);
            o.y = to_e4m3<ODD>(v(4), v(5), v(6), v(7), inv);
            turned[c8 + i][rg ^ (tid & 15)] = o;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = 32 * j + (tid >> 3), piece = 2 * (tid & 7), f = (c >> 3) & 15;
            const uint2 a = turned[c][piece ^ f], b = turned[c][(piece + 1) ^ f];
            if (kb * 128 + c < p.K)
                *reinterpret_cast<uint4*>(p.qt + (size_t)(kb * 128 + c) * p.pitch_t + (size_t)mb * 128 + 8 * piece) = uint4{a.x, a.y, b.x, b.y};
        }
    }
}

template <typename IO, int J, bool BLOCK, bool TR>
__global__ __launch_bounds__(kThreads) void quant8_kernel(QuantParams p)
{
    static_assert(J == 8 || (!BLOCK && !TR), "blocks of 128 rows and the second order take whole tiles");
    typedef Eight<IO> E;
    __shared__ uint32_t col_most[kWaves][128];
    __shared__ __align__(16) uint2 turned[TR ? 128 : 1][16];
    const int tid = (int)threadIdx.x;
    const int kb = (int)blockIdx.x % p.blocks, mb = (int)blockIdx.x / p.blocks, k0 = kb * 128 + (tid & 15) * 8, m0 = mb * 16 * J + (tid >> 4) * J;
    E raw[J];
    if (kb * 128 + 128 <= p.K) {
        // (rows behind the last are read as it, and set to zero: loads that depend on the lane would each wait for the one before)
        struct __attribute__((packed, aligned(sizeof(IO)))) Words { uint32_t w[E::W]; };
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const Words t = *reinterpret_cast<const Words*>(static_cast<const IO*>(p.x) + (size_t)min(m0 + j, p.M - 1) * p.ldx + k0);
#pragma unroll
            for (int k = 0; k < E::W; ++k) raw[j].w[k] = t.w[k];
        }
        if (mb * 16 * J + 16 * J > p.M)
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (m0 + j >= p.M)
#pragma unroll
                    for (int k = 0; k < E::W; ++k) raw[j].w[k] = 0;
    } else {
#pragma unroll
        for (int j = 0; j < J; ++j) {
#pragma unroll
            for (int k = 0; k < E::W; ++k) raw[j].w[k] = 0;
            if (m0 + j < p.M)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (k0 + i < p.K) raw[j].set(i, static_cast<const IO*>(p.x)[(size_t)(m0 + j) * p.ldx + k0 + i]);
        }
    }
    typename E::Mag most = raw[0].template magnitude<false>(0);
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int k = 0; k < E::W; ++k) most = larger(most, raw[j].template magnitude<false>(k));
    if (__syncthreads_or(E::bits(most) >= 0x7f800000u)) quant8_tile<IO, J, BLOCK, TR, true>(p, raw, col_most, turned);
    else quant8_tile<IO, J, BLOCK, TR, false>(p, raw, col_most, turned);
    // the scales' rows are filled up with zeros
    if (kb == p.blocks - 1) {
        const int rows = BLOCK ? 1 : 16 * J;
        for (int e = tid; e < rows * 3; e += kThreads) {
            const int r = mb * rows + e / 3, b = kb + 1 + e % 3;
            if (b < p.sp && (BLOCK || r < p.M)) p.s[(size_t)r * p.sp + b] = 0;
        }
    }
    if (TR && mb == p.blocks_t - 1) {
        const int rows = BLOCK ? 1 : 128;
        for (int e = tid; e < rows * 3; e += kThreads) {
            const int r = kb * rows + e / 3, b = mb + 1 + e % 3;
            if (b < p.sp_t && (BLOCK || r < p.K)) p.st[(size_t)r * p.sp_t + b] = 0;
        }
    }
}

namespace {
// Workgroups of 128 x 128 values where blocks or the second order need them, else of 16 x 128: those of 128 take as long for many rows
// (16384 x 8192 75.4 us against 74.6, 16384 x 4100 43.0 against 38.5) and longer for few (64 x 8192 3.8 us against 2.6).
bool quant_whole(bool block, bool tr) { return block || tr; }
long long quant_tiles(int M, int K, bool whole) { return ((long long)M + (whole ? 127 : 15)) / (whole ? 128 : 16) * (hgrn2_quant8_pitch(K) / 128); }

template <typename IO> hipError_t launch_quant(const QuantParams& p, bool block, hipStream_t st)
{
    const bool tr = p.qt != nullptr;
    const dim3 grid((unsigned)quant_tiles(p.M, p.K, quant_whole(block, tr)));
    if (block && tr) quant8_kernel<IO, 8, true, true><<<grid, kThreads, 0, st>>>(p);
    else if (block) quant8_kernel<IO, 8, true, false><<<grid, kThreads, 0, st>>>(p);
    else if (tr) quant8_kernel<IO, 8, false, true><<<grid, kThreads, 0, st>>>(p);
    else quant8_kernel<IO, 1, false, false><<<grid, kThreads, 0, st>>>(p);
    return hipGetLastError();
}
}   // namespace

}   // namespace hgrn2

using namespace hgrn2;

extern "C" {

int32_t hgrn2_quant8_pitch(int32_t K) { return K > 0 && K <= 0x7fffff00 ? (K + 127) / 128 * 128 : 0; }
int32_t hgrn2_quant8_scale_pitch(int32_t K) { return K > 0 && K <= 0x7fffff00 ? (int32_t)(((int64_t)K + 511) / 512 * 4) : 0; }

int hgrn2_quant8(int32_t M, int32_t K, int32_t io_dtype, const void* x, int64_t ld_x, int32_t block_rows, uint8_t* q, uint8_t* scale, uint8_t* q_t,
                 uint8_t* scale_t, void* stream)
{
    if (M < 0 || K <= 0 || K > 0x7fffff00 || M > 0x7fffff00 || (io_dtype != HGRN2_F32 && io_dtype != HGRN2_BF16) || (ld_x && ld_x < K)) return HGRN2_ERR_SHAPE;
    if (block_rows != 1 && block_rows != 128) return HGRN2_ERR_UNSUPPORTED;
    if (!launchable(quant_tiles(M, K, quant_whole(block_rows == 128, q_t != nullptr)), kThreads)) return HGRN2_ERR_UNSUPPORTED;
    if (M == 0) return HGRN2_OK;
    if (!x || !q || !scale || (q_t != nullptr) != (scale_t != nullptr)) return HGRN2_ERR_NULL;
    if (((uintptr_t)q | (uintptr_t)q_t) & 15) return HGRN2_ERR_UNSUPPORTED;
    QuantParams p{x, ld_x ? ld_x : K, M, K, hgrn2_quant8_pitch(K), hgrn2_quant8_pitch(M), hgrn2_quant8_scale_pitch(K), hgrn2_quant8_scale_pitch(M),
                  hgrn2_quant8_pitch(K) / 128, hgrn2_quant8_pitch(M) / 128, q, scale, q_t, scale_t};
    hipStream_t st = static_cast<hipStream_t>(stream);
    const hipError_t e = io_dtype == HGRN2_BF16 ? launch_quant<__bf16>(p, block_rows == 128, st) : launch_quant<float>(p, block_rows == 128, st);
    return e == hipSuccess ? HGRN2_OK : HGRN2_ERR_HIP;
}

}   // extern "C"
