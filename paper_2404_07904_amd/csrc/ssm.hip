// Selective state space scan: per channel d with S states, B_t and C_t shared by the channels of a group,
//
//     delta_t = softplus(dt_t + dt_bias)
//     h_t[s]  = exp(delta_t A[s]) h_(t-1)[s] + delta_t x_t B_t[s]
//     y_t     = (sum_s C_t[s] h_t[s] + D x_t) SiLU(z_t)
//
// and its reverse mode.  With e_t = exp(delta_t A), u_t = delta_t x_t, g_t = grad_y_t SiLU(z_t) and the state's gradient
// dh_t = C_t g_t + e_(t+1) dh_(t+1):
//     grad_C_t[s] = sum_d g_t h_t[s]            grad_B_t[s] = sum_d u_t dh_t[s]
//     q_t = sum_s B_t[s] dh_t[s]                r_t = sum_s A[s] w_t[s],  w_t = dh_t e_t h_(t-1)
//     grad_x_t = delta_t q_t + D g_t            grad_delta_t = x_t q_t + r_t
//     grad_A[s] = sum_t delta_t w_t[s]          grad_h0 = e_1 dh_1
//
// Every channel's every state has a decay of its own at every token, so there is no matrix product in it: an exponential and four
// operations per (token, channel, state) forward, an exponential and about twenty backward, against 8 and 14 bytes per (token,
// channel).  With 16 states both directions are bound by the vector unit (an exponential holds it for four operations' time), so
// the layout is the one that needs least beside the formulas:
//   a workgroup of four waves owns 64 channels of a group and walks a run of tokens in chunks; four lanes share a channel, each with
//   a quarter of its states in registers.  A chunk's x, dt (z, grad_y) rows come in once, four channels a lane, two chunks ahead (one in
//   reverse); what is needed per (token, channel) alone (softplus, gates) is formed there and left in LDS next to B_t and C_t, from where a
//   lane takes its operands.  Sums over states stay in a quad of lanes (each lane ends up with one of four tokens), results
//   leave through LDS as whole rows.
// Few channels would leave most of the chip idle: sequences are then cut into runs (ssm_plan.hpp).  A light walk from zero first
// finds every run's last state and the sum of its step sizes, all runs at once; the decay of a whole run is then one exponential per state,
// and a run's workgroup chains the runs before it (in reverse: behind it) into the state that it starts from.
// States and all sums are fp32.
// 8 x 2048 tokens of width 4096 with 16 states in bf16: 351 us forward, 981 in reverse, sums of the groups' channels 32 us; a copy of what
// they read and write takes 113 and 197 us.  The vector unit is busy for 86 and 81% of the waves' time: 31 instructions forward and 94 in reverse for
// each token and four states.  8 x 2048 tokens of width 2048 with 8 states 195 and 483 us (with the walk from zero), 8 x 1024 of width 2048 with 32 states 251 and 611.
#include "../../include/hgrn2.h"
#include "ssm_common.hpp"

namespace hgrn2 {

template <int SPL> struct FwdOps { float2 t; float b[SPL], c[SPL]; };

// Y: the outputs; otherwise the walk from zero that finds a run's last state and step sizes (and, with `saved` alone, a sweep that
// leaves the states entering the chunks).
enum SsmWalk { kSsmOut = 0, kSsmEnds = 1, kSsmSweep = 2 };

template <typename IO, int SPL, int WALK, bool GATE, bool WHOLE>
__global__ __launch_bounds__(kThreads) void ssm_fwd_kernel(SsmParams p)
{
    constexpr int CT = SPL == 8 ? 8 : 16, SP = 4 * SPL;
    __shared__ __align__(16) float2 du[2][CT][kSsmChannels];
    __shared__ __align__(16) float bc[2][2][CT][SP];
    __shared__ __align__(16) float ys[2][CT][kSsmPitch];
    const int tid = (int)threadIdx.x, lane = tid & 63, q = lane & 3, cl = (tid >> 6) * 16 + (lane >> 2), s0 = q * SPL;
    SsmItem it = ssm_item<CT>(p);
    const bool mine = cl < it.nd;
    const size_t d = (size_t)it.d0 + (mine ? cl : 0);
    float A2[SPL], h[SPL];
    load_states<SPL>(A2, p.A, d, p.S, s0);
#pragma unroll
    for (int i = 0; i < SPL; ++i) { A2[i] *= kLog2e; h[i] = 0.0f; }
    float sum = 0.0f;
    if (WALK != kSsmEnds && it.run % p.runs == 0 && p.hT) {
        // sequences without tokens end where they start
        const int from = p.seq.cu ? 0 : it.run / p.runs, to = p.seq.cu ? p.seq.B : from + 1;
        each_empty(p.seq, from, to, [&](int b) {
            float v[SPL] = {};
            if (p.h0) load_states<SPL>(v, p.h0 + (size_t)b * p.D * p.S, d, p.S, s0);
            if (mine) store_states<SPL>(v, p.hT + (size_t)b * p.D * p.S, d, p.S, s0);
        });
    }
    if (WALK == kSsmOut && p.zero_rest) ssm_zero_rest<WHOLE>(p, it, static_cast<IO*>(p.y));
    if (it.t1 <= max(it.t0, it.lo)) return;
    Place at = Place::of(p.seq, max(it.t0, it.lo));
    SsmChunks chunks = ssm_chunks_forward(it.t0, it.t1, CT);
    if (WALK == kSsmEnds) {
        // nobody asks for the state behind the last token of a sequence, nor for what was before that token's sequence began
        const Place end = Place::of(p.seq, it.t1 - 1);
        if (end.end <= it.t1) return;
        if (end.beg > it.t0) {
            chunks = ssm_chunks_to_end(it.t0, it.t1, end.beg, CT);
            at = chunks.first < end.beg ? Place::of(p.seq, max(chunks.first, it.lo)) : end;
        }
    } else if (at.beg < it.t0) {
        const int first_run = p.seq.cu ? ssm_first_run(at.beg, p.run_len) : it.run - it.run % p.runs;
        chain_before<SPL>(p, it.run, first_run, d, s0, A2, h);
    }
    int tc = chunks.first;
    const int n_chunks = chunks.count;
    const int stok = tid >> 4, sc = four_of(tid, it.nd);
    float bias[4], skip[4];
    load_row<float, 4>(p.dt_bias ? p.dt_bias + it.d0 + sc : p.A, p.dt_bias ? it.nd - sc : 0, bias);
    load_row<float, 4>(p.Dskip ? p.Dskip + it.d0 + sc : p.A, p.Dskip ? it.nd - sc : 0, skip);

    // Two chunks are on their way while one is worked on: with one, 8 x 2048 x 4096 waited for memory 180 of 480 us.
    typedef SsmStage<IO, SP, CT, WHOLE> Stage;
    Stage stage[2];
    Four<IO> xo, zo;
    bool real_o = false;
    auto leave = [&](const Stage& st, int buf) {
        if (CT * 16 >= kThreads || stok < CT) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float dl = st.real ? ssm_delta(p, st.dt[i] + bias[i]) : 0.0f;
                du[buf][stok][sc + i] = float2{dl, dl * st.x[i]};
            }
        }
#pragma unroll
        for (int k = 0; k < st.NBC; ++k) {
            const int e = tid + k * kThreads;
            if (e < 2 * CT * SP) (&bc[buf][0][0][0])[e] = st.there[k] ? (float)st.bc[k] : 0.0f;
        }
        xo = st.x; zo = st.z;
        real_o = st.real;
    };
    stage[0].template load<false, GATE>(p, it, tc);
    const int last_tc = tc + (n_chunks - 1) * CT;
    stage[1].template load<false, GATE>(p, it, min(tc + CT, last_tc));
    leave(stage[0], 0);
    __syncthreads();
    // chunk n, whose tokens lie in place `buf`, the same as n & 1
    auto step = [&](int n, auto BUF) {
        constexpr int buf = decltype(BUF)::value;
        // (always: where a request may be left out, the compiler waits for all of them.  Behind the end it is the last chunk's again)
        stage[buf].template load<false, GATE>(p, it, min(tc + 2 * CT, last_tc));
        const size_t chunk = (size_t)(it.chunk0 + (tc - it.t0) / CT);
        if (WALK != kSsmEnds && p.saved && mine) store_states<SPL>(h, p.saved + chunk * p.D * p.S, d, p.S, s0);
        auto operands = [&](int i) {
            FwdOps<SPL> o;
            o.t = du[buf][i][cl];
#pragma unroll
            for (int k = 0; k < SPL; ++k) {
                o.b[k] = bc[buf][0][i][s0 + k];
                if (WALK == kSsmOut) o.c[k] = bc[buf][1][i][s0 + k];
            }
            return o;
        };
        auto token = [&](const FwdOps<SPL>& o) {
            float acc = 0.0f;
#pragma unroll
            for (int k = 0; k < SPL; ++k) {
                const float e = __builtin_amdgcn_exp2f(o.t.x * A2[k]);
                h[k] = fmaf(e, h[k], o.t.y * o.b[k]);
                if (WALK == kSsmOut) acc = fmaf(o.c[k], h[k], acc);
            }
            if (WALK == kSsmEnds) sum += o.t.x;
            return acc;
        };
        if (at.beg < tc && at.end > tc + CT) {
            // a group of tokens' operands are on their way from LDS while the group before is worked on
            FwdOps<SPL> ops[2][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) ops[0][j] = operands(j);
#pragma unroll
            for (int i = 0; i < CT; i += 4) {
                float a[4];
                if (i + 4 < CT)
#pragma unroll
                    for (int j = 0; j < 4; ++j) ops[(i / 4 + 1) & 1][j] = operands(i + 4 + j);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < 4; ++j) a[j] = token(ops[(i / 4) & 1][j]);
                if (WALK == kSsmOut) ys[buf][i + q][cl] = quad_scatter(a[0], a[1], a[2], a[3], q);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            for (int i = 0; i < CT; ++i) {
                const int t = tc + i;
                if (t < it.lo || t >= it.t1) continue;
                at.forward_to(p.seq, t);
                if (t == at.beg) {
#pragma unroll
                    for (int k = 0; k < SPL; ++k) h[k] = 0.0f;
                    if (p.h0) load_states<SPL>(h, p.h0 + (size_t)at.b * p.D * p.S, d, p.S, s0);
                }
                float a = token(operands(i));
                if (WALK == kSsmOut) {
                    a += dpp<kQuadXor1>(a);
                    a += dpp<kQuadXor2>(a);
                    if (q == 0) ys[buf][i][cl] = a;
                }
                if (WALK != kSsmEnds && p.hT && mine && t + 1 == at.end) store_states<SPL>(h, p.hT + (size_t)at.b * p.D * p.S, d, p.S, s0);
            }
            at.forward_to(p.seq, tc + CT);
        }
        const Four<IO> xn = xo, zn = zo;
        const bool real_n = real_o;
        leave(stage[buf ^ 1], buf ^ 1);
        __syncthreads();
        if (WALK == kSsmOut && real_n) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = fmaf(skip[i], xn[i], ys[buf][stok][sc + i]);
                if (GATE) v[i] *= mixer_silu(zn[i]);
            }
            store_four<WHOLE>(static_cast<IO*>(p.y) + (size_t)(tc + stok) * p.D + it.d0 + sc, it.nd, v);
        }
        tc += CT;
    };
    for (int n = 0; n < n_chunks; n += 2) {
        step(n, std::integral_constant<int, 0>());
        if (n + 1 < n_chunks) step(n + 1, std::integral_constant<int, 1>());
    }
    if (WALK == kSsmEnds && mine) {
        store_states<SPL>(h, p.ends + (size_t)it.run * p.D * p.S, d, p.S, s0);
        if (q == 0) p.sums[(size_t)it.run * p.D + d] = sum;
    }
}

// Sums of the workgroups' shares, in order: grad_B and grad_C over a group's channel blocks, the parameters' over the runs.
struct SsmSums {
    Sequences seq;
    int D, S, G, per, total_runs, zero_rest;
    const float *part_bc, *part_a, *part_d;
    void *gB, *gC;
    float *gA, *gD, *gbias;
    long long n_bc, n_a;         // elements; the rest are 2 D
};
template <typename IO>
__global__ __launch_bounds__(kThreads) void ssm_sums_kernel(SsmSums p)
{
    long long e = (long long)blockIdx.x * kThreads + threadIdx.x;
    const int lo = p.seq.first(), hi = p.seq.last();
    if (e < p.n_bc) {
        const int row = 2 * p.S, s = (int)(e % row);
        const long long tg = e / row;
        const int t = (int)(tg / p.G);
        const bool ours = t >= lo && t < hi;
        if (!ours && !p.zero_rest) return;
        float v = 0.0f;
#pragma unroll 8
        for (int k = 0; k < (ours ? p.per : 0); ++k) v += p.part_bc[(size_t)k * p.n_bc + e];
        IO* to = static_cast<IO*>(s < p.S ? p.gB : p.gC);
        to[(size_t)tg * p.S + (s < p.S ? s : s - p.S)] = (IO)v;
        return;
    }
    e -= p.n_bc;
    if (e < p.n_a) {
        float v = 0.0f;
#pragma unroll 8
        for (int k = 0; k < p.total_runs; ++k) v += p.part_a[(size_t)k * p.n_a + e];
        p.gA[e] = v;
        return;
    }
    e -= p.n_a;
    if (e < 2 * p.D) {
        float v = 0.0f;
#pragma unroll 8
        for (int k = 0; k < p.total_runs; ++k) v += p.part_d[(size_t)k * 2 * p.D + e];
        if (e < p.D) { if (p.gD) p.gD[e] = v; }
        else if (p.gbias) p.gbias[e - p.D] = v;
    }
}

// ---- single tokens ----------------------------------------------------------------------------------------------------
// The same quads of lanes; the state is read and written once, 16 channels (1 KB at 16 states) a wave.
template <typename IO, int SPL>
__global__ __launch_bounds__(kThreads) void ssm_step_kernel(SsmParams p, float* state)
{
    const int lane = (int)threadIdx.x & 63, q = lane & 3, s0 = q * SPL;
    const long long first = ((long long)blockIdx.x * kWaves + ((int)threadIdx.x >> 6)) * 16 + (lane >> 2);
    const long long n = (long long)p.seq.B * p.D;
    const bool mine = first < n;
    const long long at = mine ? first : 0;
    const int b = (int)(at / p.D), d = (int)(at - (long long)b * p.D), g = d / (p.D / p.G);
    float A[SPL], h[SPL], Bt[SPL], Ct[SPL];
    load_states<SPL>(h, state, (size_t)at, p.S, s0);
    load_states<SPL>(A, p.A, (size_t)d, p.S, s0);
    load_row<IO, SPL>(static_cast<const IO*>(p.Bm) + (size_t)b * p.ldb + (size_t)g * p.S + s0, p.S - s0, Bt);
    load_row<IO, SPL>(static_cast<const IO*>(p.Cm) + (size_t)b * p.ldc + (size_t)g * p.S + s0, p.S - s0, Ct);
    const float x = (float)static_cast<const IO*>(p.x)[(size_t)b * p.ldx + d];
    const float v = (float)static_cast<const IO*>(p.dt)[(size_t)b * p.lddt + d] + (p.dt_bias ? p.dt_bias[d] : 0.0f);
    const float z = p.z ? (float)static_cast<const IO*>(p.z)[(size_t)b * p.ldz + d] : 0.0f;
    const float skip = p.Dskip ? p.Dskip[d] : 0.0f;
    const float dl = ssm_delta(p, v), u = dl * x;
    float acc = 0.0f;
#pragma unroll
    for (int k = 0; k < SPL; ++k) {
        h[k] = fmaf(__builtin_amdgcn_exp2f(dl * (kLog2e * A[k])), h[k], u * Bt[k]);
        acc = fmaf(Ct[k], h[k], acc);
    }
    acc += dpp<kQuadXor1>(acc);
    acc += dpp<kQuadXor2>(acc);
    if (!mine) return;
    store_states<SPL>(h, state, (size_t)at, p.S, s0);
    if (q == 0) {
        float o = fmaf(skip, x, acc);
        if (p.z) o *= mixer_silu(z);
        static_cast<IO*>(p.y)[(size_t)at] = (IO)o;
    }
}

namespace {

constexpr size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

struct SsmCheck { int rc; bool packed; SsmPlan plan; };

// Workgroups that add up the shares of grad_B and grad_C (n_bc elements) and of the parameters' gradients.
long long ssm_sums_groups(long long n_bc, const hgrn2_ssm_shape* s) { return (n_bc + (long long)s->D * s->S + 2ll * s->D + kThreads - 1) / kThreads; }

SsmCheck ssm_check(const hgrn2_ssm_shape* s, bool packed, bool whole, bool reverse = false)
{
    SsmCheck c{};
    c.packed = packed;
    if (!s) { c.rc = HGRN2_ERR_NULL; return c; }
    if (s->B < 0 || s->N < 0 || s->D <= 0 || s->S <= 0 || s->G <= 0) { c.rc = HGRN2_ERR_SHAPE; return c; }
    if (s->io_dtype != HGRN2_F32 && s->io_dtype != HGRN2_BF16) { c.rc = HGRN2_ERR_SHAPE; return c; }
    const long long most = 0x7fffffffll;
    const long long tokens = packed ? s->N : (long long)s->B * s->N;
    if (s->D % s->G != 0 || (long long)s->G * s->S > most || (long long)s->D * s->S > most || tokens > most - 64 || (long long)s->B * s->D > most - 512) { c.rc = HGRN2_ERR_SHAPE; return c; }
    if ((s->ld_x && s->ld_x < s->D) || (s->ld_dt && s->ld_dt < s->D) || (s->ld_z && s->ld_z < s->D) || (s->ld_grad_y && s->ld_grad_y < s->D) ||
        (s->ld_b && s->ld_b < (int64_t)s->G * s->S) || (s->ld_c && s->ld_c < (int64_t)s->G * s->S)) { c.rc = HGRN2_ERR_SHAPE; return c; }
    if (s->S > 32) { c.rc = HGRN2_ERR_UNSUPPORTED; return c; }
    // a chunk's rows are found with 32-bit offsets
    const long long widest = 1 << 24;
    if (s->D > widest || (long long)s->G * s->S > widest || s->ld_x > widest || s->ld_dt > widest || s->ld_z > widest || s->ld_grad_y > widest || s->ld_b > widest || s->ld_c > widest) {
        c.rc = HGRN2_ERR_UNSUPPORTED;
        return c;
    }
    c.plan = ssm_plan(s->B, s->N, s->D, s->S, s->G, packed, whole, reverse, s->io_dtype == HGRN2_F32);
    if ((long long)c.plan.total * c.plan.blocks > most) { c.rc = HGRN2_ERR_SHAPE; return c; }
    if (!launchable((long long)c.plan.total * c.plan.blocks, kThreads) || (reverse && !launchable(ssm_sums_groups(tokens * s->G * 2 * s->S, s), kThreads))) {
        c.rc = HGRN2_ERR_UNSUPPORTED;
        return c;
    }
    c.rc = HGRN2_OK;
    return c;
}

int ssm_tokens(const hgrn2_ssm_shape* s, bool packed) { return packed ? s->N : s->B * s->N; }

void ssm_fill(SsmParams& p, const hgrn2_ssm_shape* s, const SsmCheck& c, const int32_t* cu)
{
    p.seq = Sequences{cu, s->B, s->N, ssm_tokens(s, c.packed)};
    p.D = s->D; p.S = s->S; p.G = s->G;
    p.per = c.plan.blocks / s->G;
    p.run_len = c.plan.len; p.runs = c.plan.runs;
    p.chunks = (s->N + ssm_chunk(s->S) - 1) / ssm_chunk(s->S);
    p.softplus = s->softplus;
    p.zero_rest = c.packed ? s->zero_rest : 0;
    p.ldx = s->ld_x ? s->ld_x : s->D; p.lddt = s->ld_dt ? s->ld_dt : s->D; p.ldz = s->ld_z ? s->ld_z : s->D;
    p.ldg = s->ld_grad_y ? s->ld_grad_y : s->D;
    p.ldb = s->ld_b ? s->ld_b : (long long)s->G * s->S; p.ldc = s->ld_c ? s->ld_c : (long long)s->G * s->S;
}

size_t ssm_states_bytes(const hgrn2_ssm_shape* s, const SsmCheck& c) { return align256((size_t)c.plan.chunks * s->D * s->S * 4); }
size_t ssm_ends_bytes(const hgrn2_ssm_shape* s, const SsmCheck& c)
{
    return c.plan.runs > 1 ? align256((size_t)c.plan.total * s->D * s->S * 4) + align256((size_t)c.plan.total * s->D * 4) : 0;
}
size_t ssm_sums_bytes(const hgrn2_ssm_shape* s, const SsmCheck& c)
{
    return align256((size_t)(c.plan.blocks / s->G) * ssm_tokens(s, c.packed) * s->G * 2 * s->S * 4) +
           align256((size_t)c.plan.total * s->D * s->S * 4) + align256((size_t)c.plan.total * 2 * s->D * 4);
}

template <typename IO, int SPL, int WALK> hipError_t launch_fwd_as(const SsmParams& p, dim3 grid, hipStream_t st)
{
    constexpr bool MAY = WALK == kSsmOut;
    if (!ssm_whole(p)) {
        // (of these, which are rare, states of 8 take the kernels of 16: chunks are the same)
        if constexpr (SPL == 2) return launch_fwd_as<IO, 4, WALK>(p, grid, st);
        else if (MAY && p.z) ssm_fwd_kernel<IO, SPL, WALK, MAY, false><<<grid, kThreads, 0, st>>>(p);
        else ssm_fwd_kernel<IO, SPL, WALK, false, false><<<grid, kThreads, 0, st>>>(p);
    } else {
        if (MAY && p.z) ssm_fwd_kernel<IO, SPL, WALK, MAY, true><<<grid, kThreads, 0, st>>>(p);
        else ssm_fwd_kernel<IO, SPL, WALK, false, true><<<grid, kThreads, 0, st>>>(p);
    }
    return hipGetLastError();
}
template <int WALK> hipError_t launch_fwd(const SsmParams& p, const SsmCheck& c, int io, int S, hipStream_t st)
{
    const dim3 grid(c.plan.total * c.plan.blocks);
    const int k = ssm_lane_states(S);
    if (io == HGRN2_BF16) return k == 2 ? launch_fwd_as<__bf16, 2, WALK>(p, grid, st) : k == 4 ? launch_fwd_as<__bf16, 4, WALK>(p, grid, st) : launch_fwd_as<__bf16, 8, WALK>(p, grid, st);
    return k == 2 ? launch_fwd_as<float, 2, WALK>(p, grid, st) : k == 4 ? launch_fwd_as<float, 4, WALK>(p, grid, st) : launch_fwd_as<float, 8, WALK>(p, grid, st);
}
bool bad_workspace(const void* ws, size_t have, size_t need) { return need > 0 && (!ws || have < need || ((uintptr_t)ws & 255)); }

int ssm_forward(const hgrn2_ssm_shape* s, const int32_t* cu, bool packed, const void* x, const void* dt, const float* A, const void* Bm, const void* Cm,
                const float* D, const void* z, const float* dt_bias, const float* h0, void* y, float* hT, float* saved, size_t saved_bytes, bool saving,
                void* ws, size_t ws_bytes, void* stream)
{
    const bool whole = hT && hT == h0;
    const SsmCheck c = ssm_check(s, packed, whole && !packed);
    if (c.rc != HGRN2_OK) return c.rc;
    if (whole && packed) return HGRN2_ERR_UNSUPPORTED;
    const bool work = ssm_tokens(s, packed) > 0;
    if (s->B == 0 && !(packed && work && s->zero_rest)) return HGRN2_OK;
    if (!A || (work && (!x || !dt || !Bm || !Cm || !y))) return HGRN2_ERR_NULL;
    if (saving && work && bad_workspace(saved, saved_bytes, ssm_states_bytes(s, c))) return HGRN2_ERR_WORKSPACE;
    const size_t need = ssm_ends_bytes(s, c);
    if (bad_workspace(ws, ws_bytes, need)) return HGRN2_ERR_WORKSPACE;
    SsmParams p{};
    ssm_fill(p, s, c, cu);
    p.x = x; p.dt = dt; p.z = z; p.Bm = Bm; p.Cm = Cm; p.A = A; p.Dskip = D; p.dt_bias = dt_bias; p.h0 = h0;
    p.y = y; p.hT = hT; p.saved = saving ? saved : nullptr;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (need) {
        p.ends = static_cast<float*>(ws);
        p.sums = reinterpret_cast<float*>(static_cast<char*>(ws) + align256((size_t)c.plan.total * s->D * s->S * 4));
        if (launch_fwd<kSsmEnds>(p, c, s->io_dtype, s->S, st) != hipSuccess) return HGRN2_ERR_HIP;
    }
    return launch_fwd<kSsmOut>(p, c, s->io_dtype, s->S, st) == hipSuccess ? HGRN2_OK : HGRN2_ERR_HIP;
}

}   // namespace

}   // namespace hgrn2

using namespace hgrn2;

extern "C" {

size_t hgrn2_ssm_fwd_workspace_bytes(const hgrn2_ssm_shape* s, int32_t packed)
{
    const SsmCheck c = ssm_check(s, packed != 0, false);
    return c.rc == HGRN2_OK ? ssm_ends_bytes(s, c) : 0;
}

size_t hgrn2_ssm_saved_states_bytes(const hgrn2_ssm_shape* s, int32_t packed)
{
    const SsmCheck c = ssm_check(s, packed != 0, false);
    return c.rc == HGRN2_OK ? ssm_states_bytes(s, c) : 0;
}

size_t hgrn2_ssm_bwd_workspace_bytes(const hgrn2_ssm_shape* s, int32_t packed, int32_t saved)
{
    const SsmCheck c = ssm_check(s, packed != 0, false, true);
    return c.rc == HGRN2_OK ? ssm_ends_bytes(s, c) + ssm_sums_bytes(s, c) + (saved ? 0 : ssm_states_bytes(s, c)) : 0;
}

int hgrn2_ssm_fwd(const hgrn2_ssm_shape* s, const int32_t* cu, const void* x, const void* dt, const float* A, const void* Bm, const void* Cm, const float* D,
                  const void* z, const float* dt_bias, const float* h0, void* y, float* hT, void* ws, size_t ws_bytes, void* stream)
{
    return ssm_forward(s, cu, cu != nullptr, x, dt, A, Bm, Cm, D, z, dt_bias, h0, y, hT, nullptr, 0, false, ws, ws_bytes, stream);
}

int hgrn2_ssm_fwd_saving(const hgrn2_ssm_shape* s, const int32_t* cu, const void* x, const void* dt, const float* A, const void* Bm, const void* Cm,
                         const float* D, const void* z, const float* dt_bias, const float* h0, void* y, float* hT, void* saved, size_t saved_bytes, void* ws,
                         size_t ws_bytes, void* stream)
{
    return ssm_forward(s, cu, cu != nullptr, x, dt, A, Bm, Cm, D, z, dt_bias, h0, y, hT, static_cast<float*>(saved), saved_bytes, true, ws, ws_bytes, stream);
}

int hgrn2_ssm_bwd(const hgrn2_ssm_shape* s, const int32_t* cu, const void* x, const void* dt, const float* A, const void* Bm, const void* Cm, const float* D,
                  const void* z, const float* dt_bias, const float* h0, const void* saved, size_t saved_bytes, const void* grad_y, const float* grad_hT,
                  void* grad_x, void* grad_dt, float* grad_A, void* grad_B, void* grad_C, float* grad_D, void* grad_z, float* grad_dt_bias,
                  float* grad_h0, void* ws, size_t ws_bytes, void* stream)
{
    const bool packed = cu != nullptr;
    const SsmCheck c = ssm_check(s, packed, false, true);
    if (c.rc != HGRN2_OK) return c.rc;
    if (grad_h0 && grad_h0 == grad_hT) return HGRN2_ERR_UNSUPPORTED;
    const bool any = s->B > 0 || (packed && s->zero_rest), work = any && ssm_tokens(s, packed) > 0;
    if (!A || !grad_A || (work && (!x || !dt || !Bm || !Cm || !grad_y || !grad_x || !grad_dt || !grad_B || !grad_C || (z && !grad_z)))) return HGRN2_ERR_NULL;
    if (saved && work && bad_workspace(saved, saved_bytes, ssm_states_bytes(s, c))) return HGRN2_ERR_WORKSPACE;
    const size_t ends = ssm_ends_bytes(s, c), sums = ssm_sums_bytes(s, c), states = saved ? 0 : ssm_states_bytes(s, c);
    if (bad_workspace(ws, ws_bytes, ends + sums + states)) return HGRN2_ERR_WORKSPACE;
    SsmParams p{};
    ssm_fill(p, s, c, cu);
    p.x = x; p.dt = dt; p.z = z; p.Bm = Bm; p.Cm = Cm; p.A = A; p.Dskip = D; p.dt_bias = dt_bias; p.h0 = h0;
    p.g = grad_y; p.ghT = grad_hT; p.gx = grad_x; p.gdt = grad_dt; p.gz = grad_z; p.gh0 = grad_h0;
    char* at = static_cast<char*>(ws);
    auto take = [&](size_t bytes) { char* r = at; at += align256(bytes); return reinterpret_cast<float*>(r); };
    if (ends) {
        p.ends = take((size_t)c.plan.total * s->D * s->S * 4);
        p.sums = take((size_t)c.plan.total * s->D * 4);
    }
    p.part_bc = take((size_t)p.per * p.seq.T * s->G * 2 * s->S * 4);
    p.part_a = take((size_t)c.plan.total * s->D * s->S * 4);
    p.part_d = take((size_t)c.plan.total * 2 * s->D * 4);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (any) {
        if (saved) p.saved = static_cast<float*>(const_cast<void*>(saved));
        else {
            p.saved = reinterpret_cast<float*>(at);
            if (ends && launch_fwd<kSsmEnds>(p, c, s->io_dtype, s->S, st) != hipSuccess) return HGRN2_ERR_HIP;
            if (launch_fwd<kSsmSweep>(p, c, s->io_dtype, s->S, st) != hipSuccess) return HGRN2_ERR_HIP;
        }
        if (ends && launch_ssm_bwd<true>(p, c.plan.total * c.plan.blocks, s->io_dtype == HGRN2_BF16, st) != hipSuccess) return HGRN2_ERR_HIP;
        if (launch_ssm_bwd<false>(p, c.plan.total * c.plan.blocks, s->io_dtype == HGRN2_BF16, st) != hipSuccess) return HGRN2_ERR_HIP;
    }
    SsmSums r{};
    r.seq = p.seq; r.D = s->D; r.S = s->S; r.G = s->G; r.per = p.per; r.total_runs = any ? c.plan.total : 0; r.zero_rest = p.zero_rest;
    r.part_bc = p.part_bc; r.part_a = p.part_a; r.part_d = p.part_d;
    r.gB = grad_B; r.gC = grad_C; r.gA = grad_A; r.gD = grad_D; r.gbias = grad_dt_bias;
    r.n_bc = any ? (long long)p.seq.T * s->G * 2 * s->S : 0; r.n_a = (long long)s->D * s->S;
    const dim3 grid((unsigned)ssm_sums_groups(r.n_bc, s));
    if (s->io_dtype == HGRN2_BF16) ssm_sums_kernel<__bf16><<<grid, kThreads, 0, st>>>(r);
    else ssm_sums_kernel<float><<<grid, kThreads, 0, st>>>(r);
    return hipGetLastError() == hipSuccess ? HGRN2_OK : HGRN2_ERR_HIP;
}

int hgrn2_ssm_step(const hgrn2_ssm_shape* s, const void* x, const void* dt, const float* A, const void* Bm, const void* Cm, const float* D, const void* z,
                   const float* dt_bias, float* state, void* y, void* stream)
{
    const SsmCheck c = ssm_check(s, false, true);
    if (c.rc != HGRN2_OK) return c.rc;
    if (s->N != 1) return HGRN2_ERR_SHAPE;
    if (s->B == 0) return HGRN2_OK;
    const long long groups = ((long long)s->B * s->D + 16 * kWaves - 1) / (16 * kWaves);
    if (!launchable(groups, kThreads)) return HGRN2_ERR_UNSUPPORTED;
    if (!x || !dt || !A || !Bm || !Cm || !state || !y) return HGRN2_ERR_NULL;
    SsmParams p{};
    ssm_fill(p, s, c, nullptr);
    p.x = x; p.dt = dt; p.z = z; p.Bm = Bm; p.Cm = Cm; p.A = A; p.Dskip = D; p.dt_bias = dt_bias; p.y = y;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)groups);
    const int k = ssm_lane_states(s->S);
    if (s->io_dtype == HGRN2_BF16) {
        if (k == 2) ssm_step_kernel<__bf16, 2><<<grid, kThreads, 0, st>>>(p, state);
        else if (k == 4) ssm_step_kernel<__bf16, 4><<<grid, kThreads, 0, st>>>(p, state);
        else ssm_step_kernel<__bf16, 8><<<grid, kThreads, 0, st>>>(p, state);
    } else {
        if (k == 2) ssm_step_kernel<float, 2><<<grid, kThreads, 0, st>>>(p, state);
        else if (k == 4) ssm_step_kernel<float, 4><<<grid, kThreads, 0, st>>>(p, state);
        else ssm_step_kernel<float, 8><<<grid, kThreads, 0, st>>>(p, state);
    }
    return hipGetLastError() == hipSuccess ? HGRN2_OK : HGRN2_ERR_HIP;
}

}   // extern "C"
