"""Which rows a tile of the many-rows attention kernel has, on the CPU: the kernel's own index arithmetic, compiled for the host."""
import os
import subprocess

from paper_2510_02676_amd import build

PROGRAM = r"""
#include "ecfa_attend_many.h"
#include <cstdio>
#include <cstdlib>
using namespace ecfa;

int main()
{
    const int32_t n = 400, at[] = {0, 1, 31, 32, 33, 64, 200, 256, 399, 400};
    const int32_t wrong[][4] = {{200, 400, 400, 400}, {399, 400, 400, 400}, {400, 400, 400, 400}, {-5, 200, 300, 400}, {300, 100, 400, 50}, {0, 1 << 30, -1 << 30, 400},
                                {2147483647, 0, 400, 400}, {-2147483647 - 1, 2147483647, 5, 2147483647}, {128, 64, 32, 0}};
    const int32_t lens[] = {2147483647, 1000, -7};
    long inside = 0;
    for (uint32_t share : {1u, 4u, 5u, 33u, 128u}) {
        AttendArgs a{};
        a.share = share;
        a.b.n_seqs = 3;
        a.b.n_tokens = n;
        a.b.keys_max = 4096;
        a.b.kv_len = lens;
        const uint32_t tiles = n * share / MANY_ROWS + 3;      // as a call launches them
        const auto check = [&](const int32_t *starts, bool rising) {
            int32_t seen[3] = {0, 0, 0};
            a.b.q_start = starts;
            for (uint32_t s = 0; s < 3; s++) {
                const Seq sq = seq_of(a.b, s);
                const int32_t rows = sq.qn * (int32_t)share;
                for (uint32_t tile = 0; tile < tiles; tile++) {         // whatever sequence the search gives a tile, it stays inside of it
                    const int32_t row0 = first_row(a, s, tile, rows);
                    if (row0 == -1) continue;
                    const int32_t end = row0 + MANY_ROWS < rows ? row0 + MANY_ROWS : rows;
                    const int64_t t0 = sq.q0 + row0 / (int32_t)share, t1 = sq.q0 + (end - 1) / (int32_t)share;
                    if (row0 >= rows || row0 % MANY_ROWS || t0 < 0 || t1 < t0 || t1 >= n) {
                        printf("share %u starts %d %d %d %d sequence %u tile %u: rows %d .. %d, tokens %ld .. %ld\n", share, starts[0], starts[1], starts[2], starts[3], s, tile, row0, end, (long)t0,
                               (long)t1);
                        exit(1);
                    }
                    seen[s] += end - row0;
                    inside++;
                }
                if (rising && seen[s] != rows) {                        // and no row is left out
                    printf("share %u sequence %u: %d of %d rows\n", share, s, seen[s], rows);
                    exit(1);
                }
            }
        };
        for (const auto &w : wrong) check(w, false);
        for (int32_t w : at)
            for (int32_t x : at)
                for (int32_t y : at)
                    for (int32_t z : at) {
                        const int32_t starts[4] = {w, x, y, z};
                        check(starts, w <= x && x <= y && y <= z);
                    }
    }
    printf("inside: %ld\n", inside);
    return inside > 100000 ? 0 : 1;
}
"""


def test_tiles_stay_inside_of_their_sequence(tmp_path):
    """Starts that begin above 0, fall, are negative or lie beyond the rows: no tile has a row that its sequence does not have."""
    (tmp_path / "tiles.hip").write_text(PROGRAM)
    exe = str(tmp_path / "tiles")
    subprocess.run([build.HIPCC, "--offload-host-only", "-std=c++17", "-O1", "-I", build.CSRC, "-I", os.path.join(build.ROOT, "include"), str(tmp_path / "tiles.hip"), "-o", exe],
                   check=True, timeout=100)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and "inside:" in r.stdout, r.stdout + r.stderr
