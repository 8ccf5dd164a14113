// How nm_paged_attention shares its work (csrc/nm_paged_choice.h), compiled alone by tests/test_paged_choice.py with
// -fsanitize=address,undefined: over shapes, every query head of every request is in one row, with its own key head.
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include <vector>

#include "nm_paged_choice.h"

using namespace nm;

static int packed_shapes = 0, divided_shapes = 0;

static bool covers(const PagedShape& p)
{
    const PagedSplit a = paged_split(p);
    const int width = paged_width(a.pack * p.d), pack = paged_packs(p.cache_bytes, width) ? a.pack : 1;   // what the kernel does of it
    if (pack > 1) ++packed_shapes;
    if (a.workers) ++divided_shapes;
    const int rows = paged_rows(p.hk, pack, a.groups);
    bool ok = a.pack * p.d <= 256 && a.groups * 16 >= a.group && a.share >= 1 && rows % a.share == 0 && paged_sets(p.B, p.hk, a) * a.share == (long)p.B * rows &&
              (a.groups == 1 || a.pack == 1) && a.group % pack == 0;
    std::vector<int> seen(p.hq, 0);
    for (int set = 0; ok && set < rows / a.share; ++set)
        for (int member = 0; ok && member < a.share; ++member) {
            const PagedRow r = paged_row(set * a.share + member, a.group, a.groups);
            ok = r.heads >= 1;
            for (int i = 0; ok && i < r.heads; ++i) {
                const int h = r.h0 + i, key = r.g * pack + paged_part(i, a.group, pack);
                ok = h >= 0 && h < p.hq && !seen[h]++ && key == h / (p.hq / p.hk);
            }
        }
    for (int n : seen) ok = ok && n == 1;
    if (!ok)
        std::printf("FAILED B %d hq %d hk %d d %d bytes %d longest %ld strides %ld %ld: pack %d group %d groups %d share %d width %d\n", p.B, p.hq, p.hk, p.d,
                    p.cache_bytes, p.longest, (long)p.slot_stride, (long)p.head_stride, a.pack, a.group, a.groups, a.share, width);
    return ok;
}

// With arguments, five a shape (B, hq, hk, d, longest): how many key heads of an int8 cache laid out by tokens are taken as one.
int main(int argc, char** argv)
{
    for (int i = 1; i + 4 < argc; i += 5) {
        int v[5];
        for (int j = 0; j < 5; ++j) v[j] = std::atoi(argv[i + j]);
        std::printf("%d\n", paged_split({v[0], v[1], v[2], v[3], 1, (int64_t)v[2] * v[3], v[3], v[4]}).pack);
    }
    if (argc > 1) return 0;
    int bad = 0;
    for (int d = 16; d <= 256; d += 16)
        for (int hk : {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16, 20, 24, 32, 40, 64, 96})
            for (int group : {1, 2, 3, 4, 5, 6, 7, 8, 9, 12, 16, 17, 24, 32, 40})
                for (int bytes : {1, 2})
                    for (int by_head : {0, 1})
                        for (long longest : {1l, 128l, 512l, 513l, 1024l, 1025l, 4096l, 8192l, 131072l})
                            for (int B : {1, 3, 16, 48, 64, 96, 130, 700})
                                if (bad < 20) bad += !covers({B, hk * group, hk, d, bytes, by_head ? d : (int64_t)hk * d, by_head ? (int64_t)32 * d : d, longest});
    if (bad) return 1;
    if (packed_shapes < 1000 || divided_shapes < 1000) {
        std::printf("FAILED: %d packed and %d divided shapes\n", packed_shapes, divided_shapes);
        return 1;
    }
    std::printf("SANITIZE_OK\n");
    return 0;
}
