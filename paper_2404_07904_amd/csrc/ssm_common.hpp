// What the kernels of the selective scan (ssm.hip: forward walks, single tokens, sums; ssm_bwd.hip: reverse walks) share: a workgroup's channels and
// tokens, the chunks on their way, states of lanes and quads.
#pragma once
#include <type_traits>

#include "common.hpp"
#include "mixer.hpp"
#include "ssm_plan.hpp"

namespace hgrn2 {

struct SsmParams {
    Sequences seq;
    int D, S, G, per;              // per: channel blocks of a group
    int run_len, runs, chunks;     // runs of a sequence (packed: of the token axis); chunks of a sequence
    int softplus, zero_rest;       // zero_rest: rows of tokens that belong to no sequence are zeroed
    const void *x, *dt, *z, *g, *Bm, *Cm;
    long long ldx, lddt, ldz, ldg, ldb, ldc;      // row pitches in elements
    const float *A, *Dskip, *dt_bias, *h0, *ghT;
    void *y, *gx, *gdt, *gz;
    float *hT, *gh0;
    float *saved;                  // [chunk][D][S]: state entering every chunk
    float *ends, *sums;            // [run][D][S], [run][D]: from the walk from zero
    float *part_bc;                // [block of a group][T][G][2][S]
    float *part_a, *part_d;        // [run][D][S]; [run][2][D]: D, dt_bias
};

// Row pitch of results that the lanes of a quad write to rows of their own: four rows then lie in different banks.
constexpr int kSsmPitch = kSsmChannels + 16;

constexpr int kQuadXor1 = 0xB1, kQuadXor2 = 0x4E, kRor4 = 0x124, kRor8 = 0x128;
template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// Four values per lane of a quad -> lane q has the quad's sum of value q.
__device__ __forceinline__ float quad_scatter(float p0, float p1, float p2, float p3, int q)
{
    const bool odd = q & 1, high = q & 2;
    const float a = (odd ? p1 : p0) + dpp<kQuadXor1>(odd ? p0 : p1);
    const float b = (odd ? p3 : p2) + dpp<kQuadXor1>(odd ? p2 : p3);
    return (high ? b : a) + dpp<kQuadXor2>(high ? a : b);
}

__device__ __forceinline__ float ssm_softplus(float v)
{
    // max(v, 0) + log(1 + e), e = exp(-|v|) <= 1.  u = 1 + e is rounded by r = e - (u - 1), at most 2^-24 of it, and log(1 + e) = log(u) + r / u
    // to first order; 1 / u = 1 - e / 2 within a fifth, which is 2^-26 of e at most.
    const float e = __builtin_amdgcn_exp2f(-kLog2e * fabsf(v)), u = 1.0f + e, r = e - (u - 1.0f);
    return fmaxf(v, 0.0f) + fmaf(kLn2, __builtin_amdgcn_logf(u), r * fmaf(-0.5f, e, 1.0f));
}

// Which 64 channels and which tokens a workgroup has.
struct SsmItem {
    int g, nb, d0, nd;        // group, block in it, first channel, channels
    int run, t0, t1;          // tokens of the run that belong to a sequence lie in [max(t0, lo), t1)
    int lo;
    int chunk0;               // number of the run's first chunk
};
template <int CT>
__device__ __forceinline__ SsmItem ssm_item(const SsmParams& p)
{
    SsmItem it;
    const int blocks = p.G * p.per, blk = (int)(blockIdx.x % blocks);
    it.run = (int)(blockIdx.x / blocks);
    it.g = blk / p.per;
    it.nb = blk % p.per;
    const int wide = p.D / p.G;
    // (blocks of a group as equal as can be: none is narrow unless its group is)
    const int from = (int)((long long)it.nb * wide / p.per), to = (int)((long long)(it.nb + 1) * wide / p.per);
    it.d0 = it.g * wide + from;
    it.nd = to - from;
    if (p.seq.cu) {
        it.t0 = it.run * p.run_len;
        it.lo = p.seq.first();
        it.t1 = min(it.t0 + min(p.run_len, p.seq.T - it.t0), p.seq.last());
        it.chunk0 = it.t0 / CT;
    } else {
        const int b = it.run / p.runs, r = it.run % p.runs;
        it.t0 = b * p.seq.N + r * p.run_len;
        it.lo = it.t0;
        it.t1 = it.t0 + min(p.run_len, (b + 1) * p.seq.N - it.t0);
        it.chunk0 = b * p.chunks + r * p.run_len / CT;
    }
    return it;
}

// A lane's states of channel d: SPL floats at states[d][s0 ..], those behind S are 0.  (Nothing here branches by lane: the compiler would wait
// for every load where the paths meet.)
template <int SPL>
__device__ __forceinline__ void load_states(float (&v)[SPL], const float* states, size_t d, int S, int s0)
{
    if (S == 4 * SPL) {
        unpack(*reinterpret_cast<const RowVec<float, SPL>*>(states + d * S + s0), v);
    } else {
#pragma unroll
        for (int i = 0; i < SPL; ++i) {
            const float x = states[d * S + min(s0 + i, S - 1)];
            v[i] = s0 + i < S ? x : 0.0f;
        }
    }
}
template <int SPL>
__device__ __forceinline__ void store_states(const float (&v)[SPL], float* states, size_t d, int S, int s0)
{
    store_row<float, SPL>(states + d * S + s0, S == 4 * SPL ? SPL : S - s0, v);
}

// Four channels of a row as they come: two words of bf16, or four floats, in one load whatever their alignment.
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(4)));
template <typename IO> struct Four {
    u32x2_any w;
    __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
    __device__ __forceinline__ void set(int i, __bf16 v)
    {
        const uint32_t u = __builtin_bit_cast(uint16_t, v);
        w[i >> 1] = i & 1 ? (w[i >> 1] & 0xffffu) | u << 16 : (w[i >> 1] & 0xffff0000u) | u;
    }
};
template <> struct Four<float> {
    u32x4_any w;
    __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(w[i]); }
    __device__ __forceinline__ void set(int i, float v) { w[i] = __float_as_uint(v); }
};
// Channels sc .. of a block of `nd` channels, sc at most nd - 4, so that threads at the end of a row share some.  WHOLE: no block has
// fewer than four; such a one's rows repeat its last channel.  (A branch here would keep the compiler from counting the loads in flight.)
template <bool WHOLE, typename IO> __device__ __forceinline__ Four<IO> load_four(const IO* p, int nd)
{
    Four<IO> r;
    if constexpr (WHOLE) {
        r.w = *reinterpret_cast<const decltype(r.w)*>(p);
    } else {
        r.w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) r.set(i, p[min(i, nd - 1)]);
    }
    return r;
}
template <bool WHOLE, typename IO> __device__ __forceinline__ void store_four(IO* p, int nd, const float (&v)[4])
{
    if constexpr (WHOLE) {
        Four<IO> r;
        r.w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) r.set(i, (IO)v[i]);
        *reinterpret_cast<decltype(r.w)*>(p) = r.w;
    } else {
        store_row<IO, 4>(p, nd, v);
    }
}
__device__ __forceinline__ int four_of(int thread, int nd) { return min((thread & 15) * 4, max(nd - 4, 0)); }
// Rows of the run's tokens that belong to no sequence.
template <bool WHOLE, typename IO> __device__ __forceinline__ void ssm_zero_rest(const SsmParams& p, const SsmItem& it, IO* rows)
{
    const int from = it.t0, upto = from + min(p.run_len, p.seq.T - from), lo = p.seq.first(), hi = p.seq.last(), sc = four_of((int)threadIdx.x, it.nd);
    const float zeros[4] = {};
    if (!rows || (from >= lo && upto <= hi)) return;
    for (int t = from + ((int)threadIdx.x >> 4); t < upto; t += kThreads / 16)
        if (t < lo || t >= hi) store_four<WHOLE>(rows + (size_t)t * p.D + it.d0 + sc, it.nd, zeros);
}

// What a thread holds of a chunk that is on its way: four channels of one token of each tensor, and elements of B_t, C_t.  A chunk's rows are
// found from its first, which is the same for all lanes, with 32-bit offsets that stay what they are from chunk to chunk.
template <typename IO, int SP, int CT, bool WHOLE>
struct SsmStage {
    static constexpr int NBC = (2 * CT * SP + kThreads - 1) / kThreads;
    Four<IO> x, dt, z, g;
    IO bc[NBC];
    bool real, there[NBC];
    uint32_t ox, odt, oz, og, obc[NBC];
    static __device__ __forceinline__ Four<IO> four(const IO* p, const SsmItem& it) { return load_four<WHOLE>(p, it.nd); }
    template <typename T> static __device__ __forceinline__ const T* at(const T* p, uint32_t bytes)
    {
        return reinterpret_cast<const T*>(reinterpret_cast<const char*>(p) + bytes);
    }
    __device__ __forceinline__ void offsets(const SsmParams& p, const SsmItem& it, SsmTokens in)
    {
        const int tid = (int)threadIdx.x, tok = ssm_chunk_token(tid >> 4, in), c = four_of(tid, it.nd);
        constexpr uint32_t E = sizeof(IO);
        ox = (uint32_t)tok * (uint32_t)p.ldx * E + c * E;
        odt = (uint32_t)tok * (uint32_t)p.lddt * E + c * E;
        oz = (uint32_t)tok * (uint32_t)p.ldz * E + c * E;
        og = (uint32_t)tok * (uint32_t)p.ldg * E + c * E;
        real = tid >> 4 >= in.first && tid >> 4 <= in.last;
#pragma unroll
        for (int k = 0; k < NBC; ++k) {
            const int e = tid + k * kThreads, i = e / SP % CT, s = e % SP, j = ssm_chunk_token(i, in);
            obc[k] = (uint32_t)j * (uint32_t)(e / (CT * SP) & 1 ? p.ldc : p.ldb) * E + min(s, p.S - 1) * E;
            there[k] = s < p.S && i >= in.first && i <= in.last;
        }
    }
    template <bool G, bool Z>
    __device__ __forceinline__ void load(const SsmParams& p, const SsmItem& it, int tc)
    {
        const SsmTokens in = ssm_tokens_of(tc, it.t0, it.lo, it.t1, CT);
        const bool part = in.first > 0 || in.last < CT - 1;
        if (part || changed) {
            offsets(p, it, in);
            changed = part;
        }
        x = four(at(static_cast<const IO*>(p.x) + (size_t)tc * p.ldx + it.d0, ox), it);
        dt = four(at(static_cast<const IO*>(p.dt) + (size_t)tc * p.lddt + it.d0, odt), it);
        if constexpr (Z) z = four(at(static_cast<const IO*>(p.z) + (size_t)tc * p.ldz + it.d0, oz), it);
        if constexpr (G) g = four(at(static_cast<const IO*>(p.g) + (size_t)tc * p.ldg + it.d0, og), it);
        const IO* B = static_cast<const IO*>(p.Bm) + (size_t)tc * p.ldb + (size_t)it.g * p.S;
        const IO* C = static_cast<const IO*>(p.Cm) + (size_t)tc * p.ldc + (size_t)it.g * p.S;
#pragma unroll
        for (int k = 0; k < NBC; ++k) {
            if constexpr (CT * SP == kThreads) bc[k] = *at(k ? C : B, obc[k]);
            else bc[k] = *at((int)threadIdx.x + k * kThreads >= CT * SP ? C : B, obc[k]);
        }
    }
    bool changed = true;       // (the same in every lane) the offsets are not those of a whole chunk
};

__device__ __forceinline__ float ssm_delta(const SsmParams& p, float v) { return p.softplus ? ssm_softplus(v) : v; }

// What enters a run, decayed through it, and what the run adds.  (A growth past the range of fp32 leaves a zero what it is, as token by token.)
__device__ __forceinline__ float through_run(float exponent, float in, float adds) { return in == 0.0f ? adds : fmaf(__builtin_amdgcn_exp2f(exponent), in, adds); }

// The sequences of [from, to) without tokens, 64 looked at at a time.
template <typename F> __device__ __forceinline__ void each_empty(const Sequences& s, int from, int to, F f)
{
    for (int b0 = from; b0 < to; b0 += 64) {
        const int b = b0 + ((int)threadIdx.x & 63);
        bool empty = b < to;
        if (empty && s.cu) empty = min(max(s.cu[b], 0), s.T) >= min(max(s.cu[b + 1], 0), s.T);
        else if (empty) empty = s.N == 0;
        for (unsigned long long m = __ballot(empty); m; m &= m - 1) f(b0 + __ffsll(m) - 1);
    }
}

// The state a run starts from, when it starts inside a sequence: the runs of the sequence before it applied in order.
template <int SPL>
__device__ __forceinline__ void chain_before(const SsmParams& p, int run, int first_run, size_t d, int s0, const float (&A2)[SPL], float (&h)[SPL])
{
    load_states<SPL>(h, p.ends + (size_t)first_run * p.D * p.S, d, p.S, s0);
#pragma unroll 4
    for (int k = first_run + 1; k < run; ++k) {
        float e[SPL];
        load_states<SPL>(e, p.ends + (size_t)k * p.D * p.S, d, p.S, s0);
        const float sum = p.sums[(size_t)k * p.D + d];
#pragma unroll
        for (int i = 0; i < SPL; ++i) h[i] = through_run(sum * A2[i], h[i], e[i]);
    }
}

// Whether every block of channels has four at least.
inline bool ssm_whole(const SsmParams& p) { return p.D / p.G >= 4; }

// ENDS: the walk from zero.  `io_bf16`: storage of the sequence tensors.
template <bool ENDS> hipError_t launch_ssm_bwd(const SsmParams& p, int groups, bool io_bf16, hipStream_t st);

}   // namespace hgrn2
