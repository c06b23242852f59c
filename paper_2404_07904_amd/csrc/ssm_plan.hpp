// How the selective scan cuts a batch into runs: plain host arithmetic, in a header of its own so that it can be compiled and
// checked without a GPU.
#pragma once
#include <stdint.h>

#include <cmath>

namespace hgrn2 {

constexpr int kSsmChannels = 64;      // channels of a workgroup

// States per lane (four lanes share a channel) and tokens of a chunk: registers hold a chunk's states and decays in the reverse walk.
inline int ssm_lane_states(int S) { return S <= 8 ? 2 : S <= 16 ? 4 : 8; }
inline int ssm_chunk(int S) { return S <= 16 ? 16 : 8; }

// Workgroups of a walk that a compute unit holds, by its registers and LDS (in reverse two: 8 states fit three times, but 1 x 8192 x 2048 takes 281 us
// counted so, 266 with two).
inline int ssm_held(int S, bool f32, bool reverse) { return reverse ? 2 : S <= 8 ? (f32 ? 3 : 4) : S <= 16 ? (f32 ? 2 : 3) : 2; }

struct SsmPlan {
    int blocks;       // channel blocks: groups x blocks of a group
    int len;          // tokens of a run, a multiple of 16
    int runs;         // runs of a sequence (equal lengths), or of the token axis (packed)
    int total;        // all runs
    int chunks;       // chunks of all sequences
};

// whole: sequences in one piece (equal lengths).  reverse: for the reverse walks; chunks are the same for both.  f32: storage.
inline SsmPlan ssm_plan(int B, int N, int D, int S, int G, bool packed, bool whole, bool reverse = false, bool f32 = false)
{
    SsmPlan p;
    const int per = (D / G + kSsmChannels - 1) / kSsmChannels, chunk = ssm_chunk(S);
    p.blocks = G * per;
    const long long units = (long long)p.blocks * (packed || B < 1 ? 1 : B);
    // Workgroups of four waves, three or four for each compute unit and as many as make whole rounds of those it holds: a run more costs a walk from zero over nearly all tokens, which pays from one
    // workgroup a unit on forward and from two on in reverse (where the walk from zero is a smaller part): 4 x 2048 x 4096 x 16, 256 workgroups
    // uncut, in one piece / cut: forward 243 / 259 us, reverse 767 / 663; 8 x 2048 x 1024, 128 of them, forward 143 cut in eight, 154 in four.
    const long long slots = 256 * ssm_held(S, f32, reverse), target = (1024 + slots / 2) / slots * slots;
    long long want = whole || units >= (reverse ? 512 : 256) ? 1 : target / units;
    // Runs of 64 tokens at least, or 32 where those would not give every unit one (128 tokens of width 4096: 25.0 -> 19.5 us, reverse 63 -> 49;
    // 16 x 256 x 512, where they do: 31 -> 36).
    const long long runs64 = ((long long)N + 63) / 64, most = units * runs64 <= 256 ? ((long long)N + 31) / 32 : runs64;
    if (want > most) want = most;
    // A run adds up the ends of those before it one after the other, so runs and their lengths grow together, as the root of the tokens:
    // runs at most 1.3 sqrt(N), without / with that bound: 1 x 32768 x 64 x 16 forward 110 / 76 us, reverse 161 / 136; 1 x 65536 x 128,
    // 173 / 135 and 292 / 280 (with 0.7 sqrt(N) 84 and 169; 133 and 280).
    const long long root = 1 + (long long)std::sqrt(1.7 * N);
    if (want > root) want = root;
    auto cut = [&]() {
        if (want < 1) want = 1;
        p.len = (int)((((long long)N + want - 1) / want + 15) / 16 * 16);
        if (p.len < 16) p.len = 16;
        p.runs = N > 0 ? (int)(((long long)N + p.len - 1) / p.len) : 1;
    };
    cut();
    // A last round that is less than three quarters full costs more than longer runs: 3001 packed tokens of width 1030 in fp32, 846 workgroups / 504,
    // reverse 117 / 105 us; 1 x 16384 x 256, 588 / 512, reverse 143 / 115; rounds as whole as that, 3 x 5000 x 700, 32 runs / 31, reverse 265 / 242.
    const long long rounds = (units * p.runs + slots - 1) / slots;
    if (p.runs > 1 && rounds > 1 && units * p.runs * 4 < (4 * rounds - 1) * slots) {
        want = slots * (rounds - 1) / units;
        cut();
    }
    p.total = packed ? p.runs : p.runs * B;
    p.chunks = packed ? (N + chunk - 1) / chunk : B * ((N + chunk - 1) / chunk);
    return p;
}

}   // namespace hgrn2
