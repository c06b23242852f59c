// What the operators of the selective state space mixer (conv.hip, ssm.hip) share: which sequence a token belongs to, and
// rows of any alignment.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ssm_walk.hpp"

namespace hgrn2 {

// A launch has fewer than 2^32 threads along an axis.
inline bool launchable(long long groups, int threads) { return groups < (1ll << 32) / threads; }

// Sequences on a token axis of T tokens: B of N tokens each (cu null, T = B N), or cu[b] .. cu[b + 1] - 1 for sequence b.
// Offsets of a packed batch are clamped to the token axis; a wrong array can only give wrong results: every access of a kernel is
// to a token in [0, T) that it was given, and to a sequence in [0, B).
struct Sequences {
    const int32_t* cu;
    int B, N, T;
    __device__ __forceinline__ int start(int b) const
    {
        if (!cu) return b * N;
        typedef const __attribute__((address_space(4))) int32_t* const_ptr;
        return min(max(((const_ptr)cu)[b], 0), T);
    }
    __device__ __forceinline__ int first() const { return cu ? start(0) : 0; }
    __device__ __forceinline__ int last() const { return start(B); }
};

// The sequence a wave is in as it walks along the token axis.  All values are the same in every lane.
struct Place {
    int b, beg, end;
    // the last sequence that starts at token t or before, t < s.last() (64 lanes look at 64 offsets at a time): beg <= t < end
    __device__ __forceinline__ static Place of(const Sequences& s, int t)
    {
        int b = 0;
        if (!s.cu) {
            b = s.N > 0 ? min(t / s.N, s.B - 1) : 0;
        } else {
            const int lane = (int)threadIdx.x & 63;
            int n = s.B;
            while (n > 1) {
                const int step = (n + 63) / 64, i = lane * step;
                const bool before = i < n && min(max(s.cu[b + i], 0), s.T) <= t;
                const int count = __popcll(__ballot(before));
                b += max(count - 1, 0) * step;
                n = min(step, s.B - b);
            }
            b = __builtin_amdgcn_readfirstlane(b);
        }
        Place p;
        p.b = b;
        p.beg = place_first(s.start(b), t);
        p.end = place_end(s.start(b + 1), t, s.last());
        return p;
    }
    __device__ __forceinline__ void forward_to(const Sequences& s, int t)
    {
        while (t >= end && b + 1 < s.B) {
            ++b;
            beg = end;
            end = max(s.start(b + 1), beg);
        }
    }
    __device__ __forceinline__ void back_to(const Sequences& s, int t)
    {
        while (t < beg && b > 0) {
            --b;
            end = beg;
            beg = min(s.start(b), end);
        }
    }
};

// ---- rows of any alignment: vectors that need no more alignment than their elements -------------------------------
template <typename IO, int V> struct __attribute__((packed, aligned(sizeof(IO)))) RowVec { IO e[V]; };

// V elements at p, of which n are there (others: 0): as they are, as floats
template <typename IO, int V> __device__ __forceinline__ RowVec<IO, V> raw_row(const IO* p, int n)
{
    if (n >= V) return *reinterpret_cast<const RowVec<IO, V>*>(p);
    RowVec<IO, V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) r.e[i] = i < n ? p[i] : (IO)0.0f;
    return r;
}
template <typename IO, int V> __device__ __forceinline__ void unpack(const RowVec<IO, V>& r, float (&v)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (float)r.e[i];
}
template <typename IO, int V>
__device__ __forceinline__ void load_row(const IO* p, int n, float (&out)[V])
{
    unpack(raw_row<IO, V>(p, n), out);
}
template <typename IO, int V>
__device__ __forceinline__ void store_row(IO* p, int n, const float (&v)[V])
{
    if (n >= V) {
        RowVec<IO, V> r;
#pragma unroll
        for (int i = 0; i < V; ++i) r.e[i] = (IO)v[i];
        *reinterpret_cast<RowVec<IO, V>*>(p) = r;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) p[i] = (IO)v[i];
    }
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float mixer_sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * x)); }
__device__ __forceinline__ float mixer_silu(float x) { return x * mixer_sigmoid(x); }
__device__ __forceinline__ float silu_slope(float x)
{
    const float g = mixer_sigmoid(x);
    return g * fmaf(x, 1.0f - g, 1.0f);
}

}   // namespace hgrn2
