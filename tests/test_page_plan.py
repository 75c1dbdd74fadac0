"""How the attention over pages and the selection of beams are cut into workgroups: host arithmetic and the functions that the kernels call, compiled and
swept on the CPU.  Every item is in one part, whatever the rows' lengths turn out to be; parts, grid and workspace stay bounded."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2305_13144_amd", "csrc")

PROGRAM = r"""
#include "ss_plan.h"
#include <algorithm>
#include <cstdio>
#include <random>
#include <vector>
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main()
{
    using namespace ss;
    long tried = 0;
    // plans and their workspaces
    for (int group : {1, 2, 5, 32})
        for (int groups : {1, 2, 16, 300, 2047})
            for (int n_kv : {1, 3, 8, 40})
                for (int each : {1, 4, 7, 16, 33})
                    for (int hd : {64, 128})
                        for (long long len : {0LL, 1LL, 512LL, 513LL, 1500LL, 4000LL, 1LL << 20, 2147483647LL}) {
                            const PagePlan p = page_plan(group * groups, group, n_kv, each, hd, (int)len, 256);
                            CHECK(p.tiles == 1 || p.tiles == 2);
                            CHECK((long long)p.row_blocks * 16 * p.tiles >= group * each && (long long)(p.row_blocks - 1) * 16 * p.tiles < group * each);
                            const long long units = (long long)groups * n_kv * p.row_blocks;
                            CHECK(p.parts >= 0 && p.parts <= 1024 && (p.parts <= 1 || p.parts * units <= p.at_once));
                            const PageSpace s = page_space(p, group * groups, group, n_kv, hd, 16, 300);
                            const size_t part = (size_t)16 * p.tiles * (hd + 4) * 4;
                            CHECK(s.notes % 16 == 0 && s.counts % 16 == 0 && s.items % 16 == 0 && s.bytes % 16 == 0);
                            CHECK(s.notes >= part * (p.parts == 1 ? 0 : p.parts > 1 ? units * p.parts : page_grid(p.at_once, units, group)));
                            CHECK(s.counts - s.notes >= (p.parts == 0 ? 16 + (size_t)units * 8 : 0));
                            CHECK(group == 1 ? s.bytes == s.counts : s.items - s.counts >= (size_t)groups * 4 && s.bytes - s.items == (size_t)groups * group * 300 * 16);
                            ++tried;
                        }
    // equal parts
    for (int most : {-1, 0, 1, 2, 24, 1024})
        for (int count : {0, 1, 7, 8, 9, 100, 244, 5000, 1 << 27}) {
            const int n = page_parts(count, most);
            CHECK(n >= 1 && n <= std::max(most, 1) && (n == 1 || count / n >= kPageShare));
            CHECK(page_cut(count, 0, n) == 0 && page_cut(count, n, n) == count);
            for (int k = 0; k < n; ++k) CHECK(count < n || page_cut(count, k, n) < page_cut(count, k + 1, n));
        }
    // parts by the rows' lengths
    std::mt19937 r(7);
    for (int round = 0; round < 4000; ++round) {
        const int groups = 1 + r() % 200, units = 1 + r() % 40, group = 1 + r() % 2, at_once = r() % 2 ? 768 : 512;
        const long long top = r() % 3 == 0 ? 30 : r() % 2 ? 3000 : 1 << 22;
        std::vector<int> count(groups);
        long long all = 0;
        for (int& c : count) all += c = r() % 5 == 0 ? 0 : (int)(r() % top);
        if (all == 0) continue;
        const int average = (int)std::min(std::max((all * units + at_once - 1) / at_once, (long long)kPageShare), 1LL << 28);
        for (PageCuts cuts : {page_large_cuts(average), page_least_cuts(average, group), PageCuts{0, average + 1 + average / 3}}) {
            long long parts = 0;
            for (int c : count) {
                const int n = cuts.large_of(c) + cuts.small_of(c);
                CHECK((n == 0) == (c == 0));
                parts += (long long)n * units;
                int at = 0;
                for (int k = 0; k < n; ++k) {
                    int i0, i1;
                    cuts.part(c, k, &i0, &i1);
                    CHECK(i0 == at && i1 > i0 && i1 - i0 <= std::max(cuts.large, cuts.small));
                    at = i1;
                }
                CHECK(at == c);
            }
            if (cuts.large == 0) CHECK(parts <= page_grid(at_once, (long long)groups * units, group));
        }
        ++tried;
    }
    // beams
    for (int groups : {0, 1, 7, 300, 65535})
        for (int beams : {1, 2, 8, 64})
            for (int keep : {1, 8, 64})
                for (int vocab : {1, 2, 1000, 32000, 100003, 2147483647})
                    for (int size : {2, 4}) {
                        const int s = beam_slices(groups, beams, vocab, keep, size, 256);
                        CHECK(s >= 1 && s <= beam_slices(groups, beams, vocab, keep, 4, 256));
                        CHECK(s == 1 || (long long)s * beams * keep <= kBeamRanked);
                        CHECK(s == 1 || (long long)(s - 1) * groups * beams < 512);
                        ++tried;
                    }
    std::printf("ok %ld\n", tried);
}
"""


SINGLE = r"""
#include "ss_plan.h"
#include <algorithm>
#include <cstdio>
#include <random>
#include <vector>
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
using namespace ss;
static long long parts_of(const PageCuts& c, const std::vector<int>& count, int units)
{
    long long parts = 0;
    for (int n : count) parts += (long long)(c.large_of(n) + c.small_of(n)) * units;
    return parts;
}
int main()
{
    std::mt19937 r(11);
    long tried = 0;
    for (int round = 0; round < 200000; ++round) {
        const int groups = 1 + r() % (round % 10 ? 100 : 5000), units = 1 + r() % 40, at_once = r() % 2 ? 768 : 512;
        const long long top = r() % 2 ? 6000 : 1 << (4 + r() % 23);
        std::vector<int> count(groups);
        long long all = 0;
        for (int& c : count) all += c = r() % 4 == 0 ? 0 : r() % 3 ? (int)(r() % top) : (int)top;
        auto average_of = [&](long long n) { return std::max((n * units + at_once - 1) / at_once, (long long)kPageShare); };
        if (r() % 5 == 0 && average_of(all) < 1 << 20) {   // as many items as make half a part and one more: two small parts of what is left, everywhere
            const int some = (int)average_of(all);
            all = 0;
            for (int& c : count) all += c = some * (int)(r() % 3) + some / 2 + 1;
        }
        if (all == 0 || average_of(all) > 1 << 28) continue;
        const int a = (int)average_of(all);
        const long long grid = page_grid(at_once, (long long)groups * units, 1);
        CHECK(parts_of(page_large_cuts(a), count, units) <= grid);
        CHECK(parts_of(page_least_cuts(a, 1), count, units) <= page_grid(at_once, (long long)groups * units, 2));
        ++tried;
    }
    std::printf("ok %ld\n", tried);
}
"""


def test_a_grid_has_room_for_every_part_of_single_rows(tmp_path):
    """... with the cuts that are tried first: others are never needed there."""
    src, exe = tmp_path / "single.cpp", tmp_path / "single"
    src.write_text(SINGLE)
    subprocess.run(["g++", "-std=c++17", "-O2", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.startswith("ok"), out.stdout + out.stderr


def test_every_item_is_in_one_part(tmp_path):
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-I", CSRC, str(src), os.path.join(CSRC, "ss_plan.cpp"),
                    "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.startswith("ok"), out.stdout + out.stderr
