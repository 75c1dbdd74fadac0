"""Entries of the tables that the operators on device tensors read on the GPU: what counts as inside.  The functions that the kernels call are
compiled and swept here on the CPU, with sums that overflow turned into errors; no such table reaches the GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2305_13144_amd", "csrc")


def run(tmp_path, body):
    src, exe = tmp_path / "tables.cpp", tmp_path / "tables"
    src.write_text('#include "ss_plan.h"\n#include <climits>\n#include <cstdio>\ntypedef __int128 wide;\nint main()\n{\n' + body + '    std::printf("ok\\n");\n}\n')
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-Werror", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-I", CSRC,
                    str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout == "ok\n", out.stdout + out.stderr


def test_slabs_beyond_the_cache_are_outside_wherever_they_start(tmp_path):
    run(tmp_path, r"""
    for (int64_t total : {(int64_t)0, (int64_t)1, (int64_t)80, (int64_t)INT_MAX + 5, INT64_MAX})
        for (int slots : {INT_MIN, -1, 0, 1, 30, 80, 81, INT_MAX})
            for (int64_t start : {INT64_MIN, (int64_t)-1, (int64_t)0, (int64_t)1, (int64_t)50, (int64_t)51, (int64_t)80, (int64_t)INT_MAX, INT64_MAX - INT_MAX,
                                  INT64_MAX - 30, INT64_MAX - 1, INT64_MAX}) {
                const bool want = start >= 0 && slots >= 0 && (wide)start + slots <= total;
                if (ss::slab_inside(start, slots, total) != want) {
                    std::printf("start %lld, %d slots of %lld\n", (long long)start, slots, (long long)total);
                    return 1;
                }
            }
""")


def test_rows_of_tables_that_go_down_or_lead_outside_are_none(tmp_path):
    run(tmp_path, r"""
    const int some[] = {INT_MIN, INT_MIN + 5, -1, 0, 1, 5, 79, 80, 81, INT_MAX - 1, INT_MAX};
    for (int64_t rows : {(int64_t)0, (int64_t)1, (int64_t)80, (int64_t)INT_MAX, INT64_MAX})
        for (int64_t most : {(int64_t)1, (int64_t)64, (int64_t)1024, INT64_MAX})
            for (int first : some)
                for (int end : some) {
                    wide want = (wide)end - first;
                    if (want > most) want = most;
                    if (first < 0 || want < 0 || first + want > rows) want = 0;
                    if (ss::table_rows(first, end, most, rows) != (int64_t)want) {
                        std::printf("%d to %d, at most %lld of %lld\n", first, end, (long long)most, (long long)rows);
                        return 1;
                    }
                }
""")
