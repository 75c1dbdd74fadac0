"""How the attention over a cache is cut into workgroups: host arithmetic, compiled and swept on the CPU.  Every slot is in one chunk,
whatever the device's length turns out to be; the grid and the workspace stay bounded."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2305_13144_amd", "csrc")

PROGRAM = r"""
#include "ss_plan.h"
#include <cstdio>
#include <cstdlib>
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s (n_seq %d n_kv %d rows %d len %d)\n", __LINE__, #x, n_seq, n_kv, rows, len); return 1; } } while (0)
int main()
{
    long n = 0;
    for (int n_seq : {1, 2, 7, 64, 1000, 65535})
        for (int n_kv : {1, 2, 5, 8, 32, 40, 100})
            for (int rows : {1, 2, 15, 16, 17, 32, 33, 64, 128, 129, 1000, 8192})
                for (int len : {1, 2, 255, 256, 257, 512, 767, 768, 769, 5000, 131072, 1 << 22, 2147482000}) {
                    const ss::TreePlan p = ss::tree_plan(n_seq, n_kv, rows, len, 256);
                    CHECK(p.tiles == 1 || p.tiles == 2 || p.tiles == 8);
                    CHECK((long long)p.row_blocks * 16 * p.tiles >= rows && (long long)(p.row_blocks - 1) * 16 * p.tiles < rows);
                    CHECK(p.chunk >= 256 && p.chunk % 128 == 0);
                    CHECK(p.chunks >= 1 && p.chunks <= ss::kTreeMaxChunks && (long long)p.chunk * p.chunks >= len);
                    CHECK(p.chunks == 1 || (long long)p.chunk * (p.chunks - 1) < len);
                    for (int real : {0, 1, p.chunk - 1, p.chunk, p.chunk + 1, len, 2 * p.chunk + 1, 2147483647}) {
                        const int c = ss::tree_chunks(real, p.chunk, p.chunks);
                        CHECK(c >= 1 && c <= p.chunks);
                        CHECK(c == 1 || (long long)(c - 1) * p.chunk < real);       // no chunk is empty
                        CHECK(c == p.chunks || (long long)c * p.chunk >= real);     // only the last of all may be longer
                    }
                    ++n;
                }
    uint64_t mask[4 * 2];
    const int parents[4] = {-1, 0, -1, 1};
    ss::tree_mask(parents, 4, 2, mask);
    if (mask[0] != 1 || mask[2] != 3 || mask[4] != 4 || mask[6] != 11 || mask[1] || mask[3] || mask[5] || mask[7]) return 2;
    std::printf("ok %ld\n", n);
}
"""


def test_plans_cover_every_slot(tmp_path):
    src = tmp_path / "plan.cpp"
    src.write_text(PROGRAM)
    exe = tmp_path / "plan"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-I", CSRC, str(src), os.path.join(CSRC, "ss_plan.cpp"),
                    "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.startswith("ok"), out.stdout + out.stderr
