// How nm_paged_attention shares its work, in plain C++ (no HIP header: the CPU tests compile this file alone).
#pragma once

#include <algorithm>
#include <cstdint>

namespace nm {

constexpr int kPagedWaves = 4, kPagedThreads = 64 * kPagedWaves;
constexpr int kTile = 32;                       // positions a wavefront takes at once
constexpr int kUnit = kTile * kPagedWaves;      // and a workgroup

// Elements of a head that the kernels are built for: d, or that of all heads taken as one, rounded up.
constexpr int paged_width(int elements) { return elements <= 64 ? 64 : elements <= 128 ? 128 : 256; }
// Workgroups of the kernel for heads of up to dp elements that a CU has registers for (a wavefront on each SIMD each).
constexpr int workgroups_of(int dp) { return dp <= 64 ? 3 : dp <= 128 ? 2 : 1; }
// The kernels that can take neighbouring key heads as one.
constexpr bool paged_packs(int cache_bytes, int width) { return cache_bytes == 1 && width == 128; }

struct PagedShape {
    int B, hq, hk, d;
    int cache_bytes;       // of an element
    int64_t slot_stride, head_stride;
    long longest;          // positions that a request may have
};
struct PagedSplit {
    int pack;             // neighbouring key heads that a workgroup takes as one, of int8
    int group;            // query heads of a key head, packed
    int groups;           // of up to 16 of them
    int share;            // rows that read the same lines of the cache: a team of so many workgroups of one XCD takes them side by side
    int workers;          // teams that share the units; 0: one team to a set of rows
};
// Sets of rows of all requests, a.share rows each.
inline long paged_sets(int B, int hk, const PagedSplit& a) { return (long)B * (hk / a.pack) * a.groups / a.share; }

inline PagedSplit paged_split(const PagedShape& p)
{
    PagedSplit a{1, p.hq / p.hk, (p.hq / p.hk + 15) / 16, 1, 0};
    // Rows that read the same lines: the groups of a key head, and the heads whose pieces of a slot share a line of 128 bytes (as long as
    // the other slots do not lie between them).
    auto share_rows = [&] {
        const int64_t head_bytes = a.pack * p.head_stride * p.cache_bytes;
        a.share = a.groups;
        if (head_bytes > 0 && head_bytes < 128 && a.pack * p.head_stride < p.slot_stride)
            for (int n = 2; n * head_bytes <= 128; n *= 2)
                if (p.hk / a.pack % n == 0) a.share = a.groups * n;
    };
    share_rows();
    const bool divided = p.longest > (paged_sets(p.B, p.hk, a) >= 128 ? 1024 : 512);
    // Neighbouring heads of int8 as one of up to 128 elements: whole lines, and one softmax for all their queries.  Where they are too few, rows that
    // begin and end at a second kernel's cost more (us apart and packed, requests of up to 4097 positions: 16 heads of 64, 64 requests 68 and 61, 32
    // 36 and 37, 16 25 and 27; 12 of 48, 64 requests 55 and 53, 32 34 and 37; 16 of 32 61 and 39, 16 of 16 64 and 33, which gain with 32 requests too,
    // 39 and 30, 42 and 28: the line is that of 64 for all).  Not of floating-point types, where an infinity times zero is none.
    if (divided && p.cache_bytes == 1 && p.head_stride == p.d && (long)p.B * p.hk * ((p.longest + kUnit - 1) / kUnit) >= 32 * 768) {
        while (2 * a.pack * p.d <= 128 && p.hk % (2 * a.pack) == 0 && 2 * a.group <= 16) a.pack *= 2, a.group *= 2;
        // heads of 16 or 32 that are too few, or have too many queries, to fill that width: the kernel for it takes them one by one
        if (!paged_packs(p.cache_bytes, paged_width(a.pack * p.d))) a.pack = 1, a.group = p.hq / p.hk;
        share_rows();
    }
    const long most = paged_sets(p.B, p.hk, a) * ((p.longest + kUnit - 1) / kUnit);
    // Who shares: as many workgroups as run at once (twice as many took 4 % longer at 48 ragged requests and 1 to 10 % at one of 131071).
    // Rows too short to be divided go to a workgroup each, without the second kernel: tables of up to 512 positions (heads of 128, 8 rows: 14.1 us,
    // 15.3 divided), 1024 where rows go round half of the CUs (64 rows: 20.9 and 20.2; 128: 21.9 and 25.3, 22.3 if ragged; 252 of 64: 17.1 and 24.2;
    // 12 of 64 would gain too, 12.0 and 13.9, 8 of 128 lose more, 19.7 and 15.3: the line does not look at the heads' size, so that a table of 513
    // positions or more has a workspace with few rows of any).  Where that leaves CUs without one, heads of up to 64 have eight
    // wavefronts (12 heads, 300 positions: 9.3 us, 10.3 with four; heads of 128 gain less, and lose as much at one tile, by the second four).
    if (divided) a.workers = (int)std::min(most, std::max(8l, 256l * workgroups_of(paged_width(a.pack * p.d)) / a.share));
    return a;
}

// Rows of a request (a row is a key head, packed, with up to 16 query heads of its group), and one of them: key head (packed) g, query
// heads h0 .. h0 + heads - 1.  pack: 1 where the kernel does not pack.
constexpr int paged_rows(int hk, int pack, int groups) { return hk / pack * groups; }
struct PagedRow { int g, h0, heads; };
constexpr PagedRow paged_row(int row, int group, int groups)
{
    const int g = row / groups, h0 = g * group + row % groups * 16, left = (g + 1) * group - h0;
    return PagedRow{g, h0, left < 16 ? left : 16};
}
// Which of the key heads taken as one a row's query number i belongs to.
constexpr int paged_part(int i, int group, int pack)
{
    const int part = i / (group / pack);
    return part < pack ? part : pack - 1;
}

}  // namespace nm
