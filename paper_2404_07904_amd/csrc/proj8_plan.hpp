// The tiles and shares of the 8-bit product: plain host arithmetic, in a header of its own so that it can be compiled and checked
// without a GPU.
#pragma once

namespace hgrn2 {

struct Proj8Plan { int tile, splits; };      // tile 0: the kernel for few rows

// What a product takes with tiles of 256, 128 or 64, us, fitted to 65 to 16384 rows: a workgroup has a compute unit to itself (all three fill the
// LDS with steps on their way), a start and an end that nothing hides, and steps that are slower the more units work at once.
// 256 / 128 / 64: 2048^3 26.3 / 15.2 / 28.3, 4096^3 61.5 / 95.4 / 168, 128 x 8192 x 8192 36.5 / 25.2 / 21.7, 1024 x 1024 x 16384 43.4 / 32.8 / 35.3.
// Exact sums hold the vector unit and the bf16 instructions longer: 2048^3 48.5 / 24.1 / 40.9, 4096^3 105 / 152 / 268, 128 x 8192 x 8192 157 / 68.3 / 34.5,
// 1024 x 1024 x 16384 308 / 127 / 61.2 and in four shares 93.6 / 48.5 / 77.3.
inline double proj8_time(int tile, long long groups, double steps, bool exact)
{
    const double fixed = tile == 256 ? 7.0 : tile == 128 ? 4.0 : 2.2;
    const double least = exact ? (tile == 256 ? 2.3 : tile == 128 ? 0.93 : 0.41) : tile == 256 ? 1.0 : tile == 128 ? 0.32 : 0.23;
    const double more = exact ? (tile == 256 ? 0.6 : tile == 128 ? 0.1 : 0.04) : tile == 256 ? 0.68 : tile == 128 ? 0.28 : 0.04;
    const long long rest = groups % 256;
    return 2.0 + (double)(groups / 256) * (fixed + (least + more) * steps) + (rest ? fixed + (least + more * rest / 256) * steps : 0.0);
}

// steps: blocks of 128 of the contraction; exact: for exact sums.
inline Proj8Plan plan_proj8(int M, int N, int steps, bool exact = false)
{
    if (M <= 16) return Proj8Plan{0, 1};
    Proj8Plan best{64, 1};
    double least = 1e30;
    // The kernel for few rows reads all of A for every 16 rows of B, eight blocks of the contraction at a time: 17 to 32 rows, 8192 x 2048 6.7 to 8.4 us
    // (tiles of 64: 7.2), 1024 x 1024 3.5 (5.1), 2048 x 4096 9.1 (9.8), 8192 x 8192 31.2 (16.8); 64 rows 13.0 (7.2), 4.6 (5.1), 14.6 (9.8), 52.0 (18.3).
    if (M <= 64) {
        best = Proj8Plan{0, 1};
        const double groups = (N + 15) / 16 / 512.0;
        least = 2.6 + (steps + 7) / 8 * (M <= 32 ? 0.8 + 2.6 * groups : 1.8 + 4.0 * groups);
    }
    for (int tile = 64; tile <= 256; tile *= 2) {
        const long long tiles = (((long long)M + tile - 1) / tile) * (((long long)N + tile - 1) / tile);
        for (int s = 1; s <= 16 && (s == 1 || steps >= 8 * s); s *= 2) {
            // (the shares are written and read once more, and added up by a launch of their own)
            const double mb = 4e-6 * M * (double)N * s;
            if (s > 1 && mb > 64.0) break;
            const double t = proj8_time(tile, tiles * s, (double)steps / s, exact) + (s > 1 ? 3.0 + 0.4 * mb : 0.0);
            if (t < least) { least = t; best = Proj8Plan{tile, s}; }
        }
    }
    return best;
}

}   // namespace hgrn2
