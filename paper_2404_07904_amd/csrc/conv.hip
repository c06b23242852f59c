// Short causal convolution, channel by channel, with its activation:
//
//     pre_t = bias + sum_k w[k] x_(t - K + 1 + k),     y_t = SiLU(pre_t) or pre_t
//
// The K - 1 inputs before a sequence's first token are its state (zero without one); the state behind its last token is its last
// K - 1 inputs.  Reverse mode, with g_t = grad_y_t SiLU'(pre_t):
//     grad_x_t = sum_j w[K - 1 - j] g_(t + j)        (tokens of the same sequence)
//     grad_w[k] = sum_t g_t x_(t - K + 1 + k),       grad_bias = sum_t g_t
//
// A few operations per element: bound by memory, so every row is fetched once.  A lane owns 16 bytes of channels (8 in bf16, 4 in
// fp32; in reverse 4 of either; accesses that need no more alignment than an element, so odd widths and row pitches take the same path) and a wave
// a tile of consecutive tokens, whose rows are all requested before the first is used.  In reverse a wave walks several tiles and
// keeps the K - 1 rows that two tiles share in registers, and the parameters' sums, which leave once per workgroup.
// 8 x 2048 tokens of width 4096 in bf16: 62 us forward, 4.3 TB/s of x and y; 92 us in reverse with its sums, 4.4 TB/s (a copy reaches 4.8).
// Tiles that touch a sequence's first or last tokens take a path of their own that looks at every token's place.
#include "../../include/hgrn2.h"
#include "common.hpp"
#include "mixer.hpp"

namespace hgrn2 {

struct ConvParams {
    Sequences seq;
    int D, silu;
    const void *x, *s0, *gy, *gsT;
    long long ldx, ldg;
    const float *w, *bias;
    void *y, *sT, *gx, *gs0;
    float* part;          // [share][K + 1][D]
    int blocks, tiles, tail_blocks;      // channel blocks; tiles of tokens (reverse: of a workgroup); workgroups of the states
    int span;             // reverse: tokens of a wave
    int zero_rest;        // rows of y or gx of tokens that belong to no sequence are zeroed
};

template <typename IO> constexpr int conv_v() { return 16 / (int)sizeof(IO); }
// Channels of a lane of the reverse mode: windows, gradients and sums of eight do not fit its registers (8 x 2048 x 4096 in bf16: 215 us).
constexpr int kConvBackV = 4;

// Vector `item` of a row of D channels: V of them from channel c on.  The last one of a row is moved up to end with it, so that a few channels may be
// computed twice, with the same results; only rows of fewer than V channels (not FULL) have vectors of n < V.  (Loads that depend on the lane would
// each wait for the one before.)
template <int V, bool FULL> struct ConvLane {
    int c, n;
    bool real;
    __device__ __forceinline__ ConvLane(int item, int D) : c(FULL ? min(item * V, D - V) : 0), n(FULL ? V : D), real(item * V < D) {}
};
// Tokens of a tile of the reverse mode.
constexpr int conv_tile(int K) { return K == 3 ? 9 : 8; }

// Input `by` tokens before token t of the sequence at `pl`: a row of x, or of the state.
template <typename IO, int V, int K>
__device__ __forceinline__ void input_before(const ConvParams& p, const Place& pl, int t, int by, int c, int n, float (&v)[V])
{
    const int pos = t - pl.beg - by;
    if (pos >= 0) load_row<IO, V>(static_cast<const IO*>(p.x) + (size_t)(t - by) * p.ldx + c, n, v);
    else if (p.s0) load_row<IO, V>(static_cast<const IO*>(p.s0) + ((size_t)pl.b * (K - 1) + max(K - 1 + pos, 0)) * p.D + c, n, v);
    else load_row<IO, V>(static_cast<const IO*>(p.x), 0, v);
}
// The inputs of token t's window that lie before its sequence.
template <typename IO, int V, int K>
__device__ __forceinline__ void from_state(const ConvParams& p, const Place& pl, int t, int c, int n, float (&v)[K][V])
{
    const int pos = t - pl.beg;
    if (pos >= K - 1) return;
#pragma unroll
    for (int k = 0; k < K - 1; ++k)
        if (pos < K - 1 - k) {
            // row pos + k of the state
            if (p.s0) load_row<IO, V>(static_cast<const IO*>(p.s0) + ((size_t)pl.b * (K - 1) + min(max(pos + k, 0), K - 2)) * p.D + c, n, v[k]);
            else
#pragma unroll
                for (int i = 0; i < V; ++i) v[k][i] = 0.0f;
        }
}
template <int V, int K> struct ConvTaps {
    float w[K][V], bias[V];
    __device__ __forceinline__ void load(const ConvParams& p, int c, int n)
    {
        float rows[V * K], four[4];
#pragma unroll
        for (int j = 0; j < V * K; j += 4) {
            load_row<float, 4>(p.w + (size_t)c * K + j, n * K - j, four);
#pragma unroll
            for (int i = 0; i < 4; ++i) rows[j + i] = four[i];
        }
        if (p.bias) load_row<float, V>(p.bias + c, n, bias);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (!p.bias) bias[i] = 0.0f;
#pragma unroll
            for (int k = 0; k < K; ++k) w[k][i] = rows[i * K + k];
        }
    }
};

// Rows of tokens [from, upto) that belong to no sequence.
template <typename IO, int V>
__device__ __forceinline__ void zero_rest(const ConvParams& p, void* rows, int from, int upto, int c, int n)
{
    const int lo = p.seq.first(), hi = p.seq.last();
    if (!p.zero_rest || (from >= lo && upto <= hi)) return;
    const float zeros[V] = {};
    for (int t = from; t < upto; ++t)
        if (t < lo || t >= hi) store_row<IO, V>(static_cast<IO*>(rows) + (size_t)t * p.D + c, n, zeros);
}

// The state behind sequence b: rows of x, and of the state before it where it is shorter.
template <typename IO, int V, int K, bool FULL>
__device__ __forceinline__ void final_rows(const ConvParams& p, int item)
{
    const int vecs = (p.D + V - 1) / V, b = item / vecs;
    const ConvLane<V, FULL> at_lane(item - b * vecs, p.D);
    const int c = at_lane.c, n = FULL ? V : at_lane.n;
    if (b >= p.seq.B) return;
    const int beg = p.seq.start(b), len = max(p.seq.start(b + 1) - beg, 0);
    float v[V];
#pragma unroll
    for (int r = 0; r < K - 1; ++r) {
        const int at = len - (K - 1) + r;
        if (at >= 0) load_row<IO, V>(static_cast<const IO*>(p.x) + (size_t)(beg + at) * p.ldx + c, n, v);
        else load_row<IO, V>(p.s0 ? static_cast<const IO*>(p.s0) + ((size_t)b * (K - 1) + (K - 1) + at) * p.D + c : nullptr, p.s0 ? n : 0, v);
        store_row<IO, V>(static_cast<IO*>(p.sT) + ((size_t)b * (K - 1) + r) * p.D + c, n, v);
    }
}

template <typename IO, int K, int TT, bool FULL>
__global__ __launch_bounds__(kThreads) void conv_fwd_kernel(ConvParams p)
{
    constexpr int V = conv_v<IO>();
    if ((int)blockIdx.x < p.tail_blocks) {
        final_rows<IO, V, K, FULL>(p, (int)blockIdx.x * kThreads + (int)threadIdx.x);
        return;
    }
    const int id = (int)blockIdx.x - p.tail_blocks, lane = (int)threadIdx.x & 63;
    const ConvLane<V, FULL> at_lane(id % p.blocks * 64 + lane, p.D);
    const int c = at_lane.c, n = FULL ? V : at_lane.n;
    const int tile = (id / p.blocks) * kWaves + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (tile >= p.tiles) return;
    const int t0 = tile * TT, lo = p.seq.first(), hi = p.seq.last();
    if (at_lane.real) zero_rest<IO, V>(p, p.y, t0, min(t0 + TT, p.seq.T), c, n);
    if (lo >= hi || t0 >= hi || t0 + TT <= lo) return;
    Place pl = Place::of(p.seq, max(t0, lo));
    if (!at_lane.real) return;
    ConvTaps<V, K> taps;
    const IO* x = static_cast<const IO*>(p.x) + c;
    IO* y = static_cast<IO*>(p.y) + c;
    auto out = [&](int t, float (&pre)[V]) {
        if (p.silu)
#pragma unroll
            for (int i = 0; i < V; ++i) pre[i] = mixer_silu(pre[i]);
        store_row<IO, V>(y + (size_t)t * p.D, n, pre);
    };
    if (pl.beg + K - 1 <= t0 && t0 + TT <= pl.end) {
        RowVec<IO, V> rows[TT + K - 1];
#pragma unroll
        for (int r = 0; r < TT + K - 1; ++r) rows[r] = raw_row<IO, V>(x + (size_t)(t0 - (K - 1) + r) * p.ldx, n);
        taps.load(p, c, n);
        float win[K][V];
#pragma unroll
        for (int r = 0; r < K - 1; ++r) unpack(rows[r], win[r]);
#pragma unroll
        for (int r = 0; r < TT; ++r) {
            unpack(rows[r + K - 1], win[(r + K - 1) % K]);
            float pre[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                pre[i] = taps.bias[i];
#pragma unroll
                for (int k = 0; k < K; ++k) pre[i] = fmaf(taps.w[k][i], win[(r + k) % K][i], pre[i]);
            }
            out(t0 + r, pre);
        }
    } else {
        // the same rows, those outside the tensor as its first or last, and per token what its place makes of them
        RowVec<IO, V> rows[TT + K - 1];
#pragma unroll
        for (int r = 0; r < TT + K - 1; ++r) rows[r] = raw_row<IO, V>(x + (size_t)min(max(t0 - (K - 1) + r, 0), p.seq.T - 1) * p.ldx, n);
        taps.load(p, c, n);
#pragma unroll
        for (int r = 0; r < TT; ++r) {
            const int t = t0 + r;
            if (t >= lo && t < hi) {
                pl.forward_to(p.seq, t);
                float v[K][V], pre[V];
#pragma unroll
                for (int k = 0; k < K; ++k) unpack(rows[r + k], v[k]);
                from_state<IO, V, K>(p, pl, t, c, n, v);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    pre[i] = taps.bias[i];
#pragma unroll
                    for (int k = 0; k < K; ++k) pre[i] = fmaf(taps.w[k][i], v[k][i], pre[i]);
                }
                out(t, pre);
            }
        }
    }
}

// Gradient of the state before sequence b.
template <typename IO, int V, int K, bool FULL>
__device__ __forceinline__ void state_grads(const ConvParams& p, int item)
{
    const int vecs = (p.D + V - 1) / V, b = item / vecs;
    const ConvLane<V, FULL> at_lane(item - b * vecs, p.D);
    const int c = at_lane.c, n = FULL ? V : at_lane.n;
    if (b >= p.seq.B) return;
    Place pl;
    pl.b = b;
    pl.beg = p.seq.start(b);
    pl.end = max(p.seq.start(b + 1), pl.beg);
    const int len = pl.end - pl.beg;
    ConvTaps<V, K> taps;
    taps.load(p, c, n);
    float gs[K - 1][V];
#pragma unroll
    for (int r = 0; r < K - 1; ++r) {
        // the last rows of a short sequence's state are rows of this one, moved up by its length
        const int from = r - len;
        load_row<IO, V>(p.gsT && from >= 0 ? static_cast<const IO*>(p.gsT) + ((size_t)b * (K - 1) + from) * p.D + c : nullptr, p.gsT && from >= 0 ? n : 0, gs[r]);
    }
#pragma unroll
    for (int pos = 0; pos < K - 1; ++pos) {
        if (pos >= len) break;
        const int t = pl.beg + pos;
        float pre[V], g[V], v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) pre[i] = taps.bias[i];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            input_before<IO, V, K>(p, pl, t, K - 1 - k, c, n, v);
#pragma unroll
            for (int i = 0; i < V; ++i) pre[i] = fmaf(taps.w[k][i], v[i], pre[i]);
        }
        load_row<IO, V>(static_cast<const IO*>(p.gy) + (size_t)t * p.ldg + c, n, g);
#pragma unroll
        for (int r = 0; r < K - 1; ++r)
            if (r >= pos)
#pragma unroll
                for (int i = 0; i < V; ++i) gs[r][i] = fmaf(taps.w[r - pos < 0 ? 0 : r - pos][i], p.silu ? g[i] * silu_slope(pre[i]) : g[i], gs[r][i]);
    }
#pragma unroll
    for (int r = 0; r < K - 1; ++r) store_row<IO, V>(static_cast<IO*>(p.gs0) + ((size_t)b * (K - 1) + r) * p.D + c, n, gs[r]);
}

template <typename IO, int K, bool FULL>
__global__ __launch_bounds__(kThreads, 2) void conv_bwd_kernel(ConvParams p)
{
    constexpr int V = kConvBackV, TT = conv_tile(K), H = K - 1;
    static_assert(TT % K == 0, "the rings come round with every tile");
    if ((int)blockIdx.x < p.tail_blocks) {
        state_grads<IO, V, K, FULL>(p, (int)blockIdx.x * kThreads + (int)threadIdx.x);
        return;
    }
    __shared__ __align__(16) float red[kWaves - 1][K + 1][V][64];
    const int id = (int)blockIdx.x - p.tail_blocks, lane = (int)threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const ConvLane<V, FULL> at_lane(id % p.blocks * 64 + lane, p.D);
    const int c = at_lane.c, n = FULL ? V : at_lane.n, share = id / p.blocks;
    const int lo = p.seq.first(), hi = p.seq.last();
    // the tokens of this wave: span of them, the wave's part of the workgroup's
    const long long first = ((long long)share * kWaves + wave) * p.span;
    if (at_lane.real) zero_rest<IO, V>(p, p.gx, (int)min(first, (long long)p.seq.T), (int)min(first + p.span, (long long)p.seq.T), c, n);
    const int a = (int)min(first, (long long)hi), from = max(a, lo), to = min((int)min(first + p.span, (long long)hi), hi);
    float gw[K][V], gb[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        gb[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) gw[k][i] = 0.0f;
    }
    if (from < to) {
        Place pl = Place::of(p.seq, from);
        if (at_lane.real) {
        ConvTaps<V, K> taps;
        taps.load(p, c, n);
        const IO* x = static_cast<const IO*>(p.x) + c;
        const IO* gy = static_cast<const IO*>(p.gy) + c;
        IO* gx = static_cast<IO*>(p.gx) + c;
        // the gradient of pre of one token from its K inputs
        auto through = [&](const float (&g)[V], const float (&pre)[V], float (&out)[V]) {
#pragma unroll
            for (int i = 0; i < V; ++i) out[i] = p.silu ? g[i] * silu_slope(pre[i]) : g[i];
        };
        // Rings over the tokens of a stretch of tiles, kept from tile to tile: `in` has the inputs of the window behind token t0 + r
        // (the last of them H tokens ahead of it), `ring` the gradients of pre of t0 + r .. t0 + r + H.
        bool carried = false;
        float in[K][V], ring[K][V];
        // token t0 + r + H: the gradient of its pre, and its share of the parameters' sums if it counts
        auto token = [&](int r, const float (&g)[V], bool counts) {
            float pre[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                pre[i] = taps.bias[i];
#pragma unroll
                for (int k = 0; k < K; ++k) pre[i] = fmaf(taps.w[k][i], in[(r + k) % K][i], pre[i]);
            }
            through(g, pre, ring[(r + H) % K]);
            if (counts)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    gb[i] += ring[(r + H) % K][i];
#pragma unroll
                    for (int k = 0; k < K; ++k) gw[k][i] = fmaf(ring[(r + H) % K][i], in[(r + k) % K][i], gw[k][i]);
                }
        };
        auto edge = [&](int tb, int te) {
            constexpr int E = 4;
            RowVec<IO, V> xr[E + 2 * H], gr[E + H];
#pragma unroll
            for (int r = 0; r < E + 2 * H; ++r) xr[r] = raw_row<IO, V>(x + (size_t)min(max(tb - H + r, 0), p.seq.T - 1) * p.ldx, n);
#pragma unroll
            for (int r = 0; r < E + H; ++r) gr[r] = raw_row<IO, V>(gy + (size_t)min(tb + r, p.seq.T - 1) * p.ldg, n);
            int ends[E + H], seqs[E + H];
            pl.forward_to(p.seq, tb);
            Place pe = pl;
#pragma unroll
            for (int m = 0; m < E + H; ++m) {
                const int u = tb + m;
                pe.forward_to(p.seq, u);
                ends[m] = pe.end;
                seqs[m] = pe.b;
                float v[K][V], pre[V], g[V];
#pragma unroll
                for (int k = 0; k < K; ++k) unpack(xr[m + k], v[k]);
                from_state<IO, V, K>(p, pe, u, c, n, v);
                unpack(gr[m], g);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    pre[i] = taps.bias[i];
                    if (u >= hi) g[i] = 0.0f;
#pragma unroll
                    for (int k = 0; k < K; ++k) pre[i] = fmaf(taps.w[k][i], v[k][i], pre[i]);
                }
                through(g, pre, ring[m % K]);
                if (m < E && u < te)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        gb[i] += ring[m % K][i];
#pragma unroll
                        for (int k = 0; k < K; ++k) gw[k][i] = fmaf(ring[m % K][i], v[k][i], gw[k][i]);
                    }
                if (m >= H && u - H < te) {
                    const int t = u - H, end = ends[m - H < 0 ? 0 : m - H];
                    float o[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) o[i] = 0.0f;
#pragma unroll
                    for (int j = 0; j < K; ++j)
                        if (t + j < end)
#pragma unroll
                            for (int i = 0; i < V; ++i) o[i] = fmaf(taps.w[K - 1 - j][i], ring[(m - H + j + K) % K][i], o[i]);
                    const int r = t - (end - H);
                    if (p.gsT && r >= 0) {
                        // the last K - 1 tokens are rows of the state behind the sequence
                        float gs[V];
                        load_row<IO, V>(static_cast<const IO*>(p.gsT) + ((size_t)seqs[m - H < 0 ? 0 : m - H] * H + min(r, H - 1)) * p.D + c, n, gs);
#pragma unroll
                        for (int i = 0; i < V; ++i) o[i] += gs[i];
                    }
                    store_row<IO, V>(gx + (size_t)t * p.D, n, o);
                }
            }
        };
        for (int t0 = from; t0 < to; t0 += TT) {
            pl.forward_to(p.seq, t0);
            auto inside = [&](int t) { return pl.beg + H <= t && t + TT + H <= pl.end && t + TT <= to; };
            if (inside(t0)) {
                RowVec<IO, V> xr[TT], gr[TT];
#pragma unroll
                for (int r = 0; r < TT; ++r) xr[r] = raw_row<IO, V>(x + (size_t)(t0 + H + r) * p.ldx, n);
#pragma unroll
                for (int r = 0; r < TT; ++r) gr[r] = raw_row<IO, V>(gy + (size_t)(t0 + H + r) * p.ldg, n);
                if (!carried) {
                    // tokens t0 .. t0 + H - 1, as the tile before would have left them
#pragma unroll
                    for (int k = 0; k < H; ++k) load_row<IO, V>(x + (size_t)(t0 - H + k) * p.ldx, n, in[(k + K - H) % K]);
#pragma unroll
                    for (int r = -H; r < 0; ++r) {
                        float g[V];
                        load_row<IO, V>(x + (size_t)(t0 + r + H) * p.ldx, n, in[(r + H) % K]);
                        load_row<IO, V>(gy + (size_t)(t0 + r + H) * p.ldg, n, g);
                        token(r + K, g, true);
                    }
                    carried = true;
                }
                // (tokens behind the last tile of a stretch are counted where their own turn comes)
                const bool last = inside(t0 + TT);
#pragma unroll
                for (int r = 0; r < TT; ++r) {
                    float g[V], o[V];
                    unpack(xr[r], in[(r + H) % K]);
                    unpack(gr[r], g);
                    token(r, g, r < TT - H || last);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        o[i] = 0.0f;
#pragma unroll
                        for (int j = 0; j < K; ++j) o[i] = fmaf(taps.w[K - 1 - j][i], ring[(r + j) % K][i], o[i]);
                    }
                    store_row<IO, V>(gx + (size_t)(t0 + r) * p.D, n, o);
                }
            } else {
                // tokens near a sequence's ends: four at a time, each with what its place makes of the rows
                carried = false;
                for (int t = t0; t < min(t0 + TT, to); t += 4) edge(t, min(t0 + TT, to));
            }
        }
        }
    }
    // the four waves' sums, in order
    if (wave > 0)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            red[wave - 1][K][i][lane] = gb[i];
#pragma unroll
            for (int k = 0; k < K; ++k) red[wave - 1][k][i][lane] = gw[k][i];
        }
    __syncthreads();
    if (wave == 0 && at_lane.real)
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int k = 0; k <= K; ++k) {
                float v = k < K ? gw[k < K ? k : 0][i] : gb[i];
#pragma unroll
                for (int j = 0; j < kWaves - 1; ++j) v += red[j][k][i][lane];
                if (i < n) p.part[((size_t)share * (K + 1) + k) * p.D + c + i] = v;
            }
}

// The shares' sums, in order: [share][K + 1][D] -> grad_w [D][K] and grad_bias [D].  Four waves take a quarter of the shares each.
template <int K>
__global__ __launch_bounds__(kThreads) void conv_sums_kernel(const float* part, int shares, int D, float* gw, float* gb)
{
    __shared__ float red[kWaves][64];
    const int lane = (int)threadIdx.x & 63, w = (int)threadIdx.x >> 6;
    const long long e = (long long)blockIdx.x * 64 + lane;
    float v = 0.0f;
    if (e < (long long)(K + 1) * D)
#pragma unroll 8
        for (int k = (int)((long long)shares * w / kWaves); k < (int)((long long)shares * (w + 1) / kWaves); ++k) v += part[(size_t)k * (K + 1) * D + e];
    red[w][lane] = v;
    __syncthreads();
    if (w == 0 && e < (long long)(K + 1) * D) {
        v = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
        const int k = (int)(e / D), d = (int)(e - (long long)k * D);
        if (k < K) gw[(size_t)d * K + k] = v;
        else if (gb) gb[d] = v;
    }
}

template <typename IO, int K>
__global__ __launch_bounds__(64) void conv_step_kernel(ConvParams p, void* state)
{
    constexpr int V = conv_v<IO>();
    const int vecs = (p.D + V - 1) / V;
    const long long item = (long long)blockIdx.x * 64 + threadIdx.x;
    if (item >= (long long)p.seq.B * vecs) return;
    const int b = (int)(item / vecs), c = (int)(item - (long long)b * vecs) * V, n = p.D - c;
    IO* s = static_cast<IO*>(state) + (size_t)b * (K - 1) * p.D + c;
    float v[K][V];
#pragma unroll
    for (int k = 0; k < K - 1; ++k) load_row<IO, V>(s + (size_t)k * p.D, n, v[k]);
    load_row<IO, V>(static_cast<const IO*>(p.x) + (size_t)b * p.ldx + c, n, v[K - 1]);
    ConvTaps<V, K> taps;
    taps.load(p, c, n);
    float o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        o[i] = taps.bias[i];
#pragma unroll
        for (int k = 0; k < K; ++k) o[i] = fmaf(taps.w[k][i], v[k][i], o[i]);
        if (p.silu) o[i] = mixer_silu(o[i]);
    }
#pragma unroll
    for (int k = 0; k < K - 1; ++k) store_row<IO, V>(s + (size_t)k * p.D, n, v[k + 1]);
    store_row<IO, V>(static_cast<IO*>(p.y) + (size_t)b * p.D + c, n, o);
}

namespace {

constexpr int kConvMostTaps = 4;

int conv_check(const hgrn2_conv_shape* s, bool packed)
{
    if (!s) return HGRN2_ERR_NULL;
    if (s->B < 0 || s->N < 0 || s->D <= 0 || s->K <= 0) return HGRN2_ERR_SHAPE;
    if (s->io_dtype != HGRN2_F32 && s->io_dtype != HGRN2_BF16) return HGRN2_ERR_SHAPE;
    const long long most = 0x7fffffffll, tokens = packed ? s->N : (long long)s->B * s->N;
    if (tokens > most - 64 || s->D > most - 512 || (long long)s->B * s->D > most - 512) return HGRN2_ERR_SHAPE;
    if ((s->ld_x && s->ld_x < s->D) || (s->ld_grad_y && s->ld_grad_y < s->D)) return HGRN2_ERR_SHAPE;
    if (s->K < 2 || s->K > kConvMostTaps) return HGRN2_ERR_UNSUPPORTED;
    return HGRN2_OK;
}

int conv_tokens(const hgrn2_conv_shape* s, bool packed) { return packed ? s->N : s->B * s->N; }
int conv_width(const hgrn2_conv_shape* s) { return s->io_dtype == HGRN2_BF16 ? 8 : 4; }

ConvParams conv_params(const hgrn2_conv_shape* s, const int32_t* cu, const void* x, const float* w, const float* bias, const void* s0)
{
    ConvParams p{};
    p.seq = Sequences{cu, s->B, s->N, conv_tokens(s, cu != nullptr)};
    p.D = s->D; p.silu = s->silu;
    p.x = x; p.w = w; p.bias = bias; p.s0 = s0;
    p.ldx = s->ld_x ? s->ld_x : s->D;
    p.ldg = s->ld_grad_y ? s->ld_grad_y : s->D;
    p.blocks = (s->D + 64 * conv_width(s) - 1) / (64 * conv_width(s));
    p.zero_rest = s->zero_rest;
    return p;
}

int conv_tail_blocks(const hgrn2_conv_shape* s, int v) { return (int)(((long long)s->B * ((s->D + v - 1) / v) + kThreads - 1) / kThreads); }

// Workgroups of a pass over the tokens, tiles of tt of them to a wave and a workgroup's 64 lanes v channels each, and of the states'.
long long conv_groups(const hgrn2_conv_shape* s, long long tokens, int tt, int v, bool states)
{
    const long long tiles = (tokens + tt - 1) / tt, blocks = (s->D + 64ll * v - 1) / (64ll * v);
    return (states ? conv_tail_blocks(s, v) : 0) + (tiles + kWaves - 1) / kWaves * blocks;
}
// Tokens of a wave in the reverse mode: as many tiles as leave 2048 waves, two for each vector unit, one at least, 32 at most.  Each wave fetches
// K - 1 rows more than its own and leaves a row of sums for each tap.  With 4096 / 2048 / 1024 waves, bf16, K 4: 16384 tokens of width 4096
// 97.6 / 91.7 / 108.4 us, 8192 of 2048 36.0 / 30.6 / 33.9, 2048 of 2048 15.8 / 15.7 / 16.3.
int conv_span(const hgrn2_conv_shape* s, bool packed)
{
    const long long blocks = (s->D + 64 * kConvBackV - 1) / (64 * kConvBackV);
    const int tile = conv_tile(s->K);
    const long long tiles = (long long)conv_tokens(s, packed) * blocks / 2048 / tile;
    return tile * (int)(tiles < 1 ? 1 : tiles > 32 ? 32 : tiles);
}
int conv_shares(const hgrn2_conv_shape* s, bool packed)
{
    const long long per = (long long)kWaves * conv_span(s, packed);
    return (int)((conv_tokens(s, packed) + per - 1) / per);
}

bool conv_bwd_launchable(const hgrn2_conv_shape* s, bool packed)
{
    return launchable(conv_groups(s, conv_tokens(s, packed), conv_span(s, packed), kConvBackV, true), kThreads) &&
           launchable(((s->K + 1ll) * s->D + 63) / 64, kThreads);
}

template <typename IO, int K> hipError_t launch_conv_fwd(ConvParams p, bool wide, hipStream_t st)
{
    const int tt = wide && p.D >= conv_v<IO>() ? 16 : 4;
    p.tiles = (int)(((long long)p.seq.T + tt - 1) / tt);
    const dim3 grid((unsigned)(p.tail_blocks + (p.tiles + kWaves - 1) / kWaves * p.blocks));
    if (grid.x == 0) return hipSuccess;
    const bool full = p.D >= conv_v<IO>();
    if (wide && full) conv_fwd_kernel<IO, K, 16, true><<<grid, kThreads, 0, st>>>(p);
    else if (full) conv_fwd_kernel<IO, K, 4, true><<<grid, kThreads, 0, st>>>(p);
    else conv_fwd_kernel<IO, K, 4, false><<<grid, kThreads, 0, st>>>(p);
    return hipGetLastError();
}
template <typename IO, int K> hipError_t launch_conv_bwd(const ConvParams& p, int shares, float* gw, float* gb, hipStream_t st)
{
    const dim3 grid((unsigned)(p.tail_blocks + shares * p.blocks));
    if (grid.x) {
        if (p.D >= kConvBackV) conv_bwd_kernel<IO, K, true><<<grid, kThreads, 0, st>>>(p);
        else conv_bwd_kernel<IO, K, false><<<grid, kThreads, 0, st>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    conv_sums_kernel<K><<<dim3((unsigned)(((long long)(K + 1) * p.D + 63) / 64)), kThreads, 0, st>>>(p.part, shares, p.D, gw, gb);
    return hipGetLastError();
}
template <typename IO, int K> hipError_t launch_conv_step(const ConvParams& p, void* state, hipStream_t st)
{
    const int vecs = (p.D + conv_v<IO>() - 1) / conv_v<IO>();
    conv_step_kernel<IO, K><<<dim3((unsigned)(((long long)p.seq.B * vecs + 63) / 64)), 64, 0, st>>>(p, state);
    return hipGetLastError();
}

#define CONV_KERNELS(launch, ...)                                                                                       \
    (s->io_dtype == HGRN2_BF16                                                                                          \
         ? (s->K == 2 ? launch<__bf16, 2>(__VA_ARGS__) : s->K == 3 ? launch<__bf16, 3>(__VA_ARGS__) : launch<__bf16, 4>(__VA_ARGS__)) \
         : (s->K == 2 ? launch<float, 2>(__VA_ARGS__) : s->K == 3 ? launch<float, 3>(__VA_ARGS__) : launch<float, 4>(__VA_ARGS__)))

}   // namespace

}   // namespace hgrn2

using namespace hgrn2;

extern "C" {

int hgrn2_conv_fwd(const hgrn2_conv_shape* s, const int32_t* cu, const void* x, const float* w, const float* bias, const void* state, void* y,
                   void* final_state, void* stream)
{
    const int rc = conv_check(s, cu != nullptr);
    if (rc != HGRN2_OK) return rc;
    if ((final_state && final_state == state) || (y && y == x)) return HGRN2_ERR_UNSUPPORTED;
    if (s->B == 0 && !(s->zero_rest && conv_tokens(s, cu != nullptr) > 0)) return HGRN2_OK;
    if (!w || (conv_tokens(s, cu != nullptr) > 0 && (!x || !y))) return HGRN2_ERR_NULL;
    ConvParams p = conv_params(s, cu, x, w, bias, state);
    p.y = y; p.sT = final_state;
    p.tail_blocks = final_state ? conv_tail_blocks(s, conv_width(s)) : 0;
    // Tiles of 16 tokens fetch 19 rows for them, tiles of 4 seven; the latter while the former are fewer than two waves for each vector unit (bf16,
    // tiles of 16 / 4: 2048 tokens of width 2048 12.0 / 8.3 us, 4096 of 2048 15.1 / 13.0, 4096 of 4096 17.2 / 21.8, 16384 of 2048 37.4 / 39.4).
    const bool wide = (long long)p.seq.T * p.blocks >= 32 * 1024;
    if (!launchable(conv_groups(s, p.seq.T, wide && s->D >= conv_width(s) ? 16 : 4, conv_width(s), final_state != nullptr), kThreads)) return HGRN2_ERR_UNSUPPORTED;
    const hipError_t e = CONV_KERNELS(launch_conv_fwd, p, wide, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? HGRN2_OK : HGRN2_ERR_HIP;
}

size_t hgrn2_conv_bwd_workspace_bytes(const hgrn2_conv_shape* s, int32_t packed)
{
    if (conv_check(s, packed != 0) != HGRN2_OK || !conv_bwd_launchable(s, packed != 0)) return 0;
    return ((size_t)conv_shares(s, packed != 0) * (s->K + 1) * s->D * 4 + 255) & ~(size_t)255;
}

int hgrn2_conv_bwd(const hgrn2_conv_shape* s, const int32_t* cu, const void* x, const float* w, const float* bias, const void* state, const void* grad_y,
                   const void* grad_final, void* grad_x, float* grad_w, float* grad_bias, void* grad_state, void* ws, size_t ws_bytes, void* stream)
{
    const bool packed = cu != nullptr;
    const int rc = conv_check(s, packed);
    if (rc != HGRN2_OK) return rc;
    if (grad_state && grad_state == grad_final) return HGRN2_ERR_UNSUPPORTED;
    if (!conv_bwd_launchable(s, packed)) return HGRN2_ERR_UNSUPPORTED;
    const bool work = (s->B > 0 || s->zero_rest) && conv_tokens(s, packed) > 0;
    if (!w || !grad_w || (work && (!x || !grad_y || !grad_x))) return HGRN2_ERR_NULL;
    const size_t need = hgrn2_conv_bwd_workspace_bytes(s, packed ? 1 : 0);
    if (work && (!ws || ws_bytes < need || ((uintptr_t)ws & 255))) return HGRN2_ERR_WORKSPACE;
    ConvParams p = conv_params(s, cu, x, w, bias, state);
    p.gy = grad_y; p.gsT = grad_final; p.gx = grad_x; p.gs0 = grad_state;
    p.part = static_cast<float*>(ws);
    p.blocks = (s->D + 64 * kConvBackV - 1) / (64 * kConvBackV);
    p.tail_blocks = grad_state && s->B > 0 ? conv_tail_blocks(s, kConvBackV) : 0;
    p.span = conv_span(s, packed);
    const int shares = work ? conv_shares(s, packed) : 0;
    const hipError_t e = CONV_KERNELS(launch_conv_bwd, p, shares, grad_w, grad_bias, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? HGRN2_OK : HGRN2_ERR_HIP;
}

int hgrn2_conv_step(const hgrn2_conv_shape* s, const void* x, const float* w, const float* bias, void* state, void* y, void* stream)
{
    const int rc = conv_check(s, false);
    if (rc != HGRN2_OK) return rc;
    if (s->N != 1) return HGRN2_ERR_SHAPE;
    if (s->B == 0) return HGRN2_OK;
    if (!x || !w || !state || !y) return HGRN2_ERR_NULL;
    ConvParams p = conv_params(s, nullptr, x, w, bias, nullptr);
    p.y = y;
    const hipError_t e = CONV_KERNELS(launch_conv_step, p, state, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? HGRN2_OK : HGRN2_ERR_HIP;
}

}   // extern "C"
