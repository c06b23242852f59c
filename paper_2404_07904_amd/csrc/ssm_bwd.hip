// Reverse walks of the selective scan; the formulas stand in ssm.hip.
// A chunk's states are formed anew from the saved one that enters it, and stay in registers with their decays (16 tokens; 8, without decays, where a
// lane has 8 states); the walk back over them leaves grad_B and grad_C summed over the wave's channels in LDS, then over the workgroup's as a
// share of its own in memory, which a second kernel adds up in order.  No atomics: results do not change from call to call.
#include "ssm_common.hpp"

namespace hgrn2 {

// ---- reverse mode ----------------------------------------------------------------------------------------------------
// The state's gradient entering a run from behind, when the run ends inside a sequence: the runs of the sequence behind it applied from
// the last one on.
template <int SPL>
__device__ __forceinline__ void chain_behind(const SsmParams& p, int run, int last_run, size_t d, int s0, const float (&A2)[SPL], float (&c)[SPL])
{
    load_states<SPL>(c, p.ends + (size_t)last_run * p.D * p.S, d, p.S, s0);
#pragma unroll 4
    for (int k = last_run - 1; k > run; --k) {
        float e[SPL];
        load_states<SPL>(e, p.ends + (size_t)k * p.D * p.S, d, p.S, s0);
        const float sum = p.sums[(size_t)k * p.D + d];
#pragma unroll
        for (int i = 0; i < SPL; ++i) c[i] = through_run(sum * A2[i], c[i], e[i]);
    }
}

// Four values for B and four for C in every lane, summed over the four channels of a row of lanes: lanes of bank 0, 1, 2, 3 (channels of the
// row) end up with the sums of values 2, 0, 3, 1, in b[0] and c[0].  A sum that only some banks keep leaves the others to the next
// value, so twelve additions do for eight values (against six exchanges of rows and ten additions over all lanes, 8 x 2048 x 4096 x 16 1110 us
// for 1065).  (An addition that reads its neighbours waits two steps for what it reads.)
__device__ __forceinline__ void row_sums(float (&b)[4], float (&c)[4])
{
    asm("s_nop 1\n\t"
        "v_add_f32_dpp %0, %0, %0 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
        "v_add_f32_dpp %2, %2, %2 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
        "v_add_f32_dpp %4, %4, %4 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
        "v_add_f32_dpp %6, %6, %6 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
        "v_add_f32_dpp %0, %1, %1 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
        "v_add_f32_dpp %2, %3, %3 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
        "v_add_f32_dpp %4, %5, %5 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
        "v_add_f32_dpp %6, %7, %7 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
        "v_add_f32_dpp %0, %0, %0 row_ror:4 row_mask:0xf bank_mask:0xf\n\t"
        "v_add_f32_dpp %4, %4, %4 row_ror:4 row_mask:0xf bank_mask:0xf\n\t"
        "v_add_f32_dpp %0, %2, %2 row_ror:12 row_mask:0xf bank_mask:0x5\n\t"
        "v_add_f32_dpp %4, %6, %6 row_ror:12 row_mask:0xf bank_mask:0x5\n\t"
        "s_nop 1"
        : "+v"(b[0]), "+v"(b[1]), "+v"(b[2]), "+v"(b[3]), "+v"(c[0]), "+v"(c[1]), "+v"(c[2]), "+v"(c[3]));
}

// What a lane needs of a token: delta, u, g of its channel, B and C of its states.
template <int SPL> struct TokenOps { float4 t; float b[SPL], c[SPL]; };

// ENDS: the walk from zero.
template <typename IO, int SPL, bool ENDS, bool GATE, bool WHOLE>
__global__ __launch_bounds__(kThreads, 2) void ssm_bwd_kernel(SsmParams p)
{
    constexpr int CT = SPL == 8 ? 8 : 16, SP = 4 * SPL;
    __shared__ __align__(16) float4 du[CT][kSsmChannels];              // delta, u, g, x
    __shared__ __align__(16) float2 slopes[ENDS ? 1 : CT][kSsmChannels];   // d delta / d dt; grad_y times the slope of z's activation
    __shared__ __align__(16) float own[ENDS ? 1 : 2][kThreads][4];     // a thread's sums for grad_D and grad_dt_bias: not in registers, which are full
    __shared__ __align__(16) float par[2][kSsmChannels];               // dt_bias, D
    __shared__ __align__(16) float bc[2][CT][SP];
    __shared__ __align__(16) float2 qr[ENDS ? 1 : CT][kSsmPitch];
    __shared__ __align__(16) float ys[ENDS ? 1 : CT][kSsmPitch];
    __shared__ __align__(16) float dbc[ENDS ? 1 : kWaves][2][CT * SP + 32];      // grad_B, grad_C of the wave's channels (places apart by half of the banks)
    const int tid = (int)threadIdx.x, lane = tid & 63, q = lane & 3, w = tid >> 6, cl = w * 16 + (lane >> 2), s0 = q * SPL;
    SsmItem it = ssm_item<CT>(p);
    const bool mine = cl < it.nd;
    const size_t d = (size_t)it.d0 + (mine ? cl : 0);
    float A2[SPL], c[SPL], gA[SPL];
    load_states<SPL>(A2, p.A, d, p.S, s0);
#pragma unroll
    for (int i = 0; i < SPL; ++i) { A2[i] *= kLog2e; c[i] = 0.0f; gA[i] = 0.0f; }
    float sum = 0.0f;
    if (!ENDS && it.run % p.runs == 0 && p.gh0) {
        const int from = p.seq.cu ? 0 : it.run / p.runs, to = p.seq.cu ? p.seq.B : from + 1;
        each_empty(p.seq, from, to, [&](int b) {
            float v[SPL] = {};
            if (p.ghT) load_states<SPL>(v, p.ghT + (size_t)b * p.D * p.S, d, p.S, s0);
            if (mine) store_states<SPL>(v, p.gh0 + (size_t)b * p.D * p.S, d, p.S, s0);
        });
    }
    if (!ENDS && p.zero_rest) {
        ssm_zero_rest<WHOLE>(p, it, static_cast<IO*>(p.gx));
        ssm_zero_rest<WHOLE>(p, it, static_cast<IO*>(p.gdt));
        ssm_zero_rest<WHOLE>(p, it, static_cast<IO*>(p.gz));
    }
    const int from = max(it.t0, it.lo);
    const bool empty = it.t1 <= from;
    const int stok = tid >> 4, sc = four_of(tid, it.nd);
    if constexpr (!ENDS)
        for (int i = 0; i < 4; ++i) own[0][tid][i] = own[1][tid][i] = 0.0f;
    if (!empty) {
    Place at = Place::of(p.seq, it.t1 - 1);
    if (ENDS) {
        const Place start = Place::of(p.seq, from);
        if (start.beg >= from) return;               // the run's first token begins a sequence: nothing of it reaches the runs before
        if (start.end < it.t1) {                     // only the tokens of that sequence do
            it.t1 = ssm_end_back(it.t1, start.end);
            at = start;
        }
    } else if (at.end > it.t1) {
        const int last_run = p.seq.cu ? ssm_last_run(at.end, p.run_len) : it.run - it.run % p.runs + p.runs - 1;
        chain_behind<SPL>(p, it.run, last_run, d, s0, A2, c);
    }
    const SsmChunks chunks = ssm_chunks_back(it.t0, it.lo, it.t1, CT);
    const int stop = chunks.first, n_chunks = chunks.count, chunk_stop = it.chunk0 + (stop - it.t0) / CT;
    if (tid < 2 * kSsmChannels) {
        const float* from = tid < kSsmChannels ? p.dt_bias : p.Dskip;
        const int ch = tid % kSsmChannels;
        par[tid / kSsmChannels][ch] = from && ch < it.nd ? from[it.d0 + ch] : 0.0f;
    }
    SsmStage<IO, SP, CT, WHOLE> st;
    int tc = stop + (n_chunks - 1) * CT;
    st.template load<true, GATE>(p, it, tc);
    if (it.nd < kSsmChannels)
        for (int e = tid; e < CT * kSsmChannels; e += kThreads) (&du[0][0])[e] = float4{};
    __syncthreads();
    float h_next[SPL];
    if (!ENDS) load_states<SPL>(h_next, p.saved + (size_t)(chunk_stop + n_chunks - 1) * p.D * p.S, d, p.S, s0);
    for (int n = n_chunks - 1; n >= 0; --n, tc -= CT) {
        const bool real = st.real;
        if (CT * 16 >= kThreads || stok < CT)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float raw = st.dt[i] + par[0][sc + i], x = st.x[i], gy = st.g[i];
                const float dl = real ? ssm_delta(p, raw) : 0.0f;
                float g = gy, slope = 0.0f;
                if constexpr (GATE) {
                    const float z = st.z[i], sig = mixer_sigmoid(z);
                    g *= z * sig;
                    slope = gy * sig * fmaf(z, 1.0f - sig, 1.0f);
                }
                // (channels behind the block's last have none of it in the sums over channels; tokens outside the run neither)
                const bool in = real && sc + i < it.nd;
                du[stok][sc + i] = in ? float4{dl, dl * x, g, x} : float4{};
                if constexpr (!ENDS) slopes[stok][sc + i] = float2{p.softplus ? mixer_sigmoid(raw) : 1.0f, slope};
            }
#pragma unroll
        for (int k = 0; k < st.NBC; ++k) {
            const int e = tid + k * kThreads;
            if (e < 2 * CT * SP) (&bc[0][0][0])[e] = st.there[k] ? (float)st.bc[k] : 0.0f;
        }
        __syncthreads();
        st.template load<true, GATE>(p, it, max(tc - CT, stop));        // (always, as in the forward walk)
        if constexpr (ENDS) {
            auto back = [&](int i) {
                const float4 o = du[i][cl];
#pragma unroll
                for (int k = 0; k < SPL; ++k) c[k] = fmaf(bc[1][i][s0 + k], o.z, c[k]) * __builtin_amdgcn_exp2f(o.x * A2[k]);
                sum += o.x;
            };
            if (at.beg < tc && at.end > tc + CT) {
#pragma unroll
                for (int i = CT - 1; i >= 0; --i) back(i);
            } else {
                for (int i = CT - 1; i >= 0; --i) {
                    const int t = tc + i;
                    if (t < it.lo || t >= it.t1) continue;
                    at.back_to(p.seq, t);
                    if (t + 1 == at.end) {
#pragma unroll
                        for (int k = 0; k < SPL; ++k) c[k] = 0.0f;
                        if (p.ghT) load_states<SPL>(c, p.ghT + (size_t)at.b * p.D * p.S, d, p.S, s0);
                    }
                    back(i);
                }
                at.back_to(p.seq, tc - 1);
            }
            __syncthreads();
        } else {
            // (with 8 states a lane the decays are formed anew on the way back: kept, they cost 80 registers' way through scratch, 8 x 1024 x 2048 x 32
            // 688 us against 648)
            constexpr bool KEEP = SPL < 8;
            float h_in[SPL], hs[CT][SPL], a[KEEP ? CT : 1][SPL];
#pragma unroll
            for (int k = 0; k < SPL; ++k) h_in[k] = h_next[k];
            load_states<SPL>(h_next, p.saved + (size_t)(chunk_stop + max(n - 1, 0)) * p.D * p.S, d, p.S, s0);
            auto walk = [&](auto EDGE) {
                constexpr bool edge = decltype(EDGE)::value;
                uint32_t firsts = 0, lasts = 0, real_tokens = 0;
                if (edge) {
                    Place pl = at;
                    for (int i = CT - 1; i >= 0; --i) {
                        const int t = tc + i;
                        if (t < it.lo || t >= it.t1) continue;
                        pl.back_to(p.seq, t);
                        real_tokens |= 1u << i;
                        firsts |= (t == pl.beg ? 1u : 0u) << i;
                        lasts |= (t + 1 == pl.end ? 1u : 0u) << i;
                    }
                }
                Place pl = at;
                if (edge) pl.back_to(p.seq, max(tc, it.lo));
                float h[SPL], ya[4];
#pragma unroll
                for (int k = 0; k < SPL; ++k) h[k] = h_in[k];
                // a token's operands are fetched from LDS while the one before is worked on, and not earlier: registers are full of
                // the chunk's states and decays
                auto operands = [&](int i) {
                    TokenOps<SPL> r;
                    r.t = du[i][cl];
#pragma unroll
                    for (int k = 0; k < SPL; ++k) { r.b[k] = bc[0][i][s0 + k]; r.c[k] = bc[1][i][s0 + k]; }
                    return r;
                };
                TokenOps<SPL> ops = operands(0);
                // the chunk's states and decays once more
#pragma unroll
                for (int i = 0; i < CT; ++i) {
                    if (edge && (firsts >> i & 1)) {
                        pl.forward_to(p.seq, tc + i);
#pragma unroll
                        for (int k = 0; k < SPL; ++k) h[k] = 0.0f;
                        if (p.h0) load_states<SPL>(h, p.h0 + (size_t)pl.b * p.D * p.S, d, p.S, s0);
                    }
                    const TokenOps<SPL> o = ops;
                    if (i + 1 < CT) ops = operands(i + 1);
                    __builtin_amdgcn_sched_barrier(0);
                    float acc = 0.0f;
#pragma unroll
                    for (int k = 0; k < SPL; ++k) {
                        const float e = __builtin_amdgcn_exp2f(o.t.x * A2[k]);
                        if (KEEP) a[KEEP ? i : 0][k] = e;
                        h[k] = fmaf(e, h[k], o.t.y * o.b[k]);
                        hs[i][k] = h[k];
                        if (GATE) acc = fmaf(o.c[k], h[k], acc);
                    }
                    ya[i & 3] = acc;
                    if (GATE && (i & 3) == 3) ys[i - 3 + q][cl] = quad_scatter(ya[0], ya[1], ya[2], ya[3], q);
                }
                pl = at;
                ops = operands(CT - 1);
                float qa[2], ra[2], odd_row = 0.0f;
#pragma unroll
                for (int i = CT - 1; i >= 0; --i) {
                    if (edge && (lasts >> i & 1)) {
                        pl.back_to(p.seq, tc + i);
#pragma unroll
                        for (int k = 0; k < SPL; ++k) c[k] = 0.0f;
                        if (p.ghT) load_states<SPL>(c, p.ghT + (size_t)pl.b * p.D * p.S, d, p.S, s0);
                    }
                    float before[SPL];
#pragma unroll
                    for (int k = 0; k < SPL; ++k) before[k] = i > 0 ? hs[i > 0 ? i - 1 : 0][k] : h_in[k];
                    if (edge && (firsts >> i & 1)) {
                        pl.back_to(p.seq, tc + i);
#pragma unroll
                        for (int k = 0; k < SPL; ++k) before[k] = 0.0f;
                        if (p.h0) load_states<SPL>(before, p.h0 + (size_t)pl.b * p.D * p.S, d, p.S, s0);
                    }
                    const TokenOps<SPL> o = ops;
                    if (i > 0) ops = operands(i - 1);
                    __builtin_amdgcn_sched_barrier(0);
                    float qs = 0.0f, rs = 0.0f, vb[SPL], vc[SPL];
#pragma unroll
                    for (int k = 0; k < SPL; ++k) {
                        const float dh = fmaf(o.c[k], o.t.z, c[k]);
                        c[k] = dh * (KEEP ? a[KEEP ? i : 0][k] : __builtin_amdgcn_exp2f(o.t.x * A2[k]));
                        vc[k] = o.t.z * hs[i][k];
                        vb[k] = o.t.y * dh;
                        qs = fmaf(o.b[k], dh, qs);
                        // (a token of no sequence has a step of zero, but may stand next to a state that is infinite)
                        const float wk = !edge || (real_tokens >> i & 1) ? c[k] * before[k] : 0.0f;
                        rs = fmaf(A2[k], wk, rs);
                        gA[k] = fmaf(o.t.x, wk, gA[k]);
                    }
                    if (edge && (firsts >> i & 1) && p.gh0 && mine) store_states<SPL>(c, p.gh0 + (size_t)pl.b * p.D * p.S, d, p.S, s0);
                    // over the 16 channels of the wave: within the rows of lanes, then halves trade B's sums for C's, and rows trade an even
                    // token's for the odd one's (with 8 states a lane: four states' for the others'; with 2: one's for the other's, before the rows' sums)
                    if constexpr (SPL >= 4) {
                        float row[SPL / 4];
#pragma unroll
                        for (int j = 0; j < SPL / 4; ++j) {
                            float vb4[4], vc4[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) { vb4[k] = vb[(4 * j + k) % SPL]; vc4[k] = vc[(4 * j + k) % SPL]; }
                            row_sums(vb4, vc4);
                            const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(vb4[0]), __float_as_uint(vc4[0]), false, false);
                            row[j] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
                        }
                        const int bank = lane >> 2 & 3, state = s0 + (bank & 1 ? 0 : 2) + (bank >> 1), odd = lane >> 4 & 1;
                        if constexpr (SPL == 8) {
                            const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(row[0]), __float_as_uint(row[SPL / 4 - 1]), false, false);
                            dbc[w][lane >> 5][i * SP + state + 4 * odd] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
                        } else if (i & 1) {
                            odd_row = row[0];
                        } else {
                            const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(row[0]), __float_as_uint(odd_row), false, false);
                            dbc[w][lane >> 5][(i + odd) * SP + state] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
                        }
                    } else {
                        float two[2];
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(vb[j]), __float_as_uint(vc[j]), false, false);
                            two[j] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
                        }
                        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(two[0]), __float_as_uint(two[1]), false, false);
                        float v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
                        v += dpp<kRor8>(v);
                        v += dpp<kRor4>(v);
                        dbc[w][lane >> 5][i * SP + s0 + (lane >> 4 & 1)] = v;
                    }
                    qa[i & 1] = qs;
                    ra[i & 1] = rs;
                    // lane 0: q of the even token, 1: its r, 2: q of the odd one, 3: its r
                    if (!(i & 1)) reinterpret_cast<float*>(&qr[i + (q >> 1)][cl])[q & 1] = quad_scatter(qa[0], ra[0], qa[1], ra[1], q);
                }
            };
            if (at.beg < tc && at.end > tc + CT) {
                walk(std::false_type());
            } else {
                walk(std::true_type());
                at.back_to(p.seq, tc - 1);
            }
            __syncthreads();
            if (real) {
                float vx[4], vt[4], vz[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 o = qr[stok][sc + i], f2 = slopes[stok][sc + i];
                    const float4 f = du[stok][sc + i];
                    const float skip = par[1][sc + i];
                    vx[i] = fmaf(f.x, o.x, skip * f.z);
                    vt[i] = fmaf(f.w, o.x, kLn2 * o.y) * f2.x;          // (r was summed with A log2 e)
                    vz[i] = GATE ? f2.y * fmaf(skip, f.w, ys[stok][sc + i]) : 0.0f;
                    own[0][tid][i] = fmaf(f.z, f.w, own[0][tid][i]);
                    own[1][tid][i] += vt[i];
                }
                const size_t row = (size_t)(tc + stok) * p.D + it.d0 + sc;
                store_four<WHOLE>(static_cast<IO*>(p.gx) + row, it.nd, vx);
                store_four<WHOLE>(static_cast<IO*>(p.gdt) + row, it.nd, vt);
                if (GATE) {
                    store_four<WHOLE>(static_cast<IO*>(p.gz) + row, it.nd, vz);
                }
            }
            for (int e = tid; e < 2 * CT * SP; e += kThreads) {
                const int kind = e / (CT * SP), i = e / SP % CT, s = e % SP, t = tc + i;
                if (s < p.S && t >= it.lo && t < it.t1) {
                    float v = 0.0f;
#pragma unroll
                    for (int k = 0; k < kWaves; ++k) v += dbc[k][kind][i * SP + s];
                    p.part_bc[(((size_t)it.nb * p.seq.T + t) * p.G + it.g) * 2 * p.S + kind * p.S + s] = v;
                }
            }
            // (du: a thread reads and writes its own four places of it outside the walks, so the next chunk needs no barrier here)
        }
    }
    }
    if constexpr (ENDS) {
        if (mine && !empty) {
            store_states<SPL>(c, p.ends + (size_t)it.run * p.D * p.S, d, p.S, s0);
            if (q == 0) p.sums[(size_t)it.run * p.D + d] = sum;
        }
    } else {
        if (mine) store_states<SPL>(gA, p.part_a + (size_t)it.run * p.D * p.S, d, p.S, s0);
        // the threads' sums over their tokens: those of a channel are 16 threads apart
        __syncthreads();
        if (tid < 2 * kSsmChannels) {
            const int which = tid / kSsmChannels, ch = tid % kSsmChannels, col = ch >> 2;
            float v = 0.0f;
            if (ch < it.nd) {
#pragma unroll
                for (int i = 0; i < CT; ++i) v += own[which][16 * i + col][ch - four_of(col, it.nd)];
                p.part_d[((size_t)it.run * 2 + which) * p.D + it.d0 + ch] = v;
            }
        }
    }
}

namespace {
template <typename IO, int SPL, bool ENDS> hipError_t launch_bwd_as(const SsmParams& p, dim3 grid, hipStream_t st)
{
    if (!ssm_whole(p)) {
        // (of these, which are rare, states of 8 take the kernels of 16: chunks are the same)
        if constexpr (SPL == 2) return launch_bwd_as<IO, 4, ENDS>(p, grid, st);
        else if (p.z) ssm_bwd_kernel<IO, SPL, ENDS, true, false><<<grid, kThreads, 0, st>>>(p);
        else ssm_bwd_kernel<IO, SPL, ENDS, false, false><<<grid, kThreads, 0, st>>>(p);
    } else {
        if (p.z) ssm_bwd_kernel<IO, SPL, ENDS, true, true><<<grid, kThreads, 0, st>>>(p);
        else ssm_bwd_kernel<IO, SPL, ENDS, false, true><<<grid, kThreads, 0, st>>>(p);
    }
    return hipGetLastError();
}
}   // namespace

template <bool ENDS> hipError_t launch_ssm_bwd(const SsmParams& p, int groups, bool io_bf16, hipStream_t st)
{
    const dim3 grid((unsigned)groups);
    const int k = ssm_lane_states(p.S);
    if (io_bf16) return k == 2 ? launch_bwd_as<__bf16, 2, ENDS>(p, grid, st) : k == 4 ? launch_bwd_as<__bf16, 4, ENDS>(p, grid, st) : launch_bwd_as<__bf16, 8, ENDS>(p, grid, st);
    return k == 2 ? launch_bwd_as<float, 2, ENDS>(p, grid, st) : k == 4 ? launch_bwd_as<float, 4, ENDS>(p, grid, st) : launch_bwd_as<float, 8, ENDS>(p, grid, st);
}
template hipError_t launch_ssm_bwd<true>(const SsmParams&, int, bool, hipStream_t);
template hipError_t launch_ssm_bwd<false>(const SsmParams&, int, bool, hipStream_t);

}   // namespace hgrn2
