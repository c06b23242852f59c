"""Which rows, chunks and runs the walks of the selective scan touch (csrc/ssm_walk.hpp and ssm_plan.hpp, compiled here by the host compiler, no GPU
needed): packed offsets that fall, repeat, are negative or too large, and whichever sequence is taken for the one that holds a token, lead to rows of the
tensors, chunks of the saved states and runs of the workspace; offsets that rise are what they say."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2404_07904_amd", "csrc")
CHECK = r"""
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
#include "ssm_plan.hpp"
#include "ssm_walk.hpp"
using namespace hgrn2;
static long long walks = 0, chained = 0;
#define MUST(c) do { if (!(c)) { std::printf("%s: T %d run %d of %d x %d, chunk %d, b %d %d, forward %d\n", #c, T, run, p.runs, p.len, CT, b1, b2, forward); std::exit(1); } } while (0)

struct Batch {
    int T, CT;
    SsmPlan p;
    std::vector<int> cu;
    bool every;          // any sequence for any token, or the one that the search finds
    int start(int b) const { return std::min(std::max(cu[b], 0), T); }
    int lo() const { return start(0); }
    int hi() const { return start((int)cu.size() - 1); }
    int beg(int b, int t) const { return place_first(start(b), t); }
    int end(int b, int t) const { return place_end(start(b + 1), t, hi()); }
    std::vector<int> choices(int t) const
    {
        std::vector<int> r;
        const int B = (int)cu.size() - 1;
        if (every) for (int b = 0; b < B; ++b) r.push_back(b);
        else {
            int b = 0, n = B;         // 64 offsets at a time, as a wave does
            while (n > 1) {
                const int step = (n + 63) / 64;
                int count = 0;
                for (int l = 0; l < 64; ++l) count += l * step < n && start(b + l * step) <= t;
                b += std::max(count - 1, 0) * step;
                n = std::min(step, B - b);
            }
            r.push_back(b);
        }
        return r;
    }
    void rows(int run, int t0, int t1, SsmChunks c, bool states, int forward, int b1, int b2) const
    {
        ++walks;
        MUST(c.count >= 1 && c.first >= t0 && (c.first - t0) % CT == 0 && c.first < t1);
        for (int n = 0; n <= c.count; ++n) {                     // (one more is requested: the last or the first again)
            const int tc = forward ? std::min(c.first + n * CT, c.first + (c.count - 1) * CT) : std::max(c.first + (c.count - 1 - n) * CT, c.first);
            const SsmTokens in = ssm_tokens_of(tc, t0, lo(), t1, CT);
            for (int i = 0; i < CT; ++i) {
                const int tok = ssm_chunk_token(i, in);
                MUST(tok >= 0 && tok < CT && tc + tok >= 0 && tc + tok < T);
                if (i >= in.first && i <= in.last) MUST(tok == i && tc + i >= std::max(t0, lo()) && tc + i < t1 && t1 <= std::min(hi(), t0 + p.len));
            }
            const int chunk = t0 / CT + (tc - t0) / CT;
            if (states) MUST(chunk >= 0 && chunk < p.chunks);
        }
    }
    void check(int run, bool reverse) const
    {
        const int t0 = run * p.len, t1 = std::min(t0 + std::min(p.len, T - t0), hi()), from = std::max(t0, lo());
        if (t1 <= from) return;
        for (int b1 : choices(from))
            for (int b2 : choices(t1 - 1)) {
                const int forward = !reverse;
                MUST(beg(b1, from) >= 0 && beg(b1, from) <= from && end(b1, from) > from && end(b1, from) <= std::max(hi(), from + 1) && end(b1, from) <= T);
                if (!reverse) {
                    rows(run, t0, t1, ssm_chunks_forward(t0, t1, CT), true, 1, b1, b2);
                    if (beg(b1, from) < t0) {
                        const int k = ssm_first_run(beg(b1, from), p.len);
                        ++chained;
                        MUST(p.runs > 1 && k >= 0 && k < run);
                    }
                    if (end(b2, t1 - 1) > t1) {
                        SsmChunks c = ssm_chunks_forward(t0, t1, CT);
                        if (beg(b2, t1 - 1) > t0) c = ssm_chunks_to_end(t0, t1, beg(b2, t1 - 1), CT);
                        MUST(p.runs > 1 && std::max(c.first, lo()) < hi());
                        rows(run, t0, t1, c, false, 1, b1, b2);
                    }
                } else {
                    rows(run, t0, t1, ssm_chunks_back(t0, lo(), t1, CT), true, 0, b1, b2);
                    MUST(std::max(t0, lo()) < ssm_chunks_back(t0, lo(), t1, CT).first + CT);
                    if (end(b2, t1 - 1) > t1) {
                        const int k = ssm_last_run(end(b2, t1 - 1), p.len);
                        ++chained;
                        MUST(p.runs > 1 && k >= run && k < p.runs);
                    }
                    if (beg(b1, from) < from) {
                        const int cut = ssm_end_back(t1, end(b1, from));
                        MUST(cut > from && cut <= t1);
                        rows(run, t0, cut, ssm_chunks_back(t0, lo(), cut, CT), false, 0, b1, b2);
                    }
                }
            }
    }
};

int main()
{
    std::mt19937 gen(7);
    auto any = [&](int lo, int hi) { return lo + (int)(gen() % (unsigned)(hi - lo + 1)); };
    for (int trial = 0; trial < 30000; ++trial) {
        Batch b;
        b.T = any(1, trial % 3 ? 200 : 20);
        const int B = trial % 10 == 0 ? any(60, 300) : any(1, 6), S = trial % 2 ? 16 : 32;
        b.CT = ssm_chunk(S);
        const int kind = any(0, 4);
        for (int i = 0; i <= B; ++i) b.cu.push_back(kind == 0 ? any(-20, b.T + 40) : any(0, b.T));
        if (kind == 1) std::sort(b.cu.begin(), b.cu.end());
        if (kind == 2) { std::sort(b.cu.begin(), b.cu.end()); std::swap(b.cu[any(0, B)], b.cu[any(0, B)]); }
        if (kind == 3 && b.cu[0] > b.cu[B]) std::swap(b.cu[0], b.cu[B]);
        b.every = trial % 4 == 0 && B <= 6;
        for (bool reverse : {false, true}) {
            b.p = ssm_plan(B, b.T, 64, S, 1, true, false, reverse, false);
            if (trial % 5 == 1 && b.T > 16) {                   // runs of any length that a plan may have
                b.p.len = 16 * any(1, (b.T + 15) / 16);
                b.p.runs = (b.T + b.p.len - 1) / b.p.len;
            }
            for (int run = 0; run < b.p.runs; ++run) b.check(run, reverse);
        }
        if (kind == 1 && !b.every)                              // offsets that rise: the sequence that holds a token is found as it is
            for (int t = b.lo(); t < b.hi(); ++t) {
                const int c = b.choices(t)[0];
                if (!(b.cu[c] <= t && t < b.cu[c + 1] && b.beg(c, t) == b.cu[c] && b.end(c, t) == b.cu[c + 1])) { std::puts("search"); return 1; }
            }
    }
    // examples whose walks once left their tensors
    for (std::vector<int> cu : {std::vector<int>{0, 90, 10, 100}, {0, 90, 10, 20, 30, 100}, {0, 50, 20}, {100, 0}, {64, 64, 10, 64}}) {
        Batch b;
        b.cu = cu; b.T = 100; b.CT = 16; b.every = true;
        for (int len : {16, 32, 112}) {
            b.p = ssm_plan((int)cu.size() - 1, 100, 64, 16, 1, true, false);
            b.p.len = len; b.p.runs = (100 + len - 1) / len;
            for (int run = 0; run < b.p.runs; ++run) { b.check(run, false); b.check(run, true); }
        }
    }
    std::printf("ok %lld %lld\n", walks, chained);
}
"""


def test_rows_chunks_and_runs_of_any_offsets(tmp_path):
    (tmp_path / "check.cpp").write_text(CHECK)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=signed-integer-overflow", "-fno-sanitize-recover", "-static-libubsan",
                           "-I" + CSRC, str(tmp_path / "check.cpp"), "-o", str(tmp_path / "check")])
    got = subprocess.check_output([str(tmp_path / "check")], text=True).split()
    assert got[0] == "ok" and int(got[1]) > 100000 and int(got[2]) > 1000, got
