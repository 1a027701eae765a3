"""The search that a wave makes with 64 questions at once (csrc/k_probe.h), on the host: every place of every length is found, also where sums are
equal or none of them passes, and the rounds end."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2004_08532_amd", "csrc")

PROGRAM = r"""
#include <stdio.h>

#include "k_probe.h"

static int64_t find(int64_t n, int64_t first, int* rounds) {  // places first .. n - 1 hold
    Probes p = {0, n - 1};
    *rounds = 0;
    while (p.open() && *rounds < 100) {
        int lane = 0;
        while (lane < 63 && p.at(lane) < first) ++lane;
        if (p.at(63) != p.hi || p.at(0) < p.lo) return -2;
        p.narrow(lane);
        ++*rounds;
    }
    return p.lo == p.hi ? p.lo : -1;
}

int main() {
    int bad = 0, rounds, most = 0;
    for (int64_t n = 1; n <= 5000; ++n)
        for (int64_t first = 0; first <= n; first += n < 700 || first + 130 > n ? 1 : 3) {
            const int64_t got = find(n, first, &rounds);
            if (rounds > most) most = rounds;
            if (got != (first < n ? first : n - 1) && bad++ < 20) printf("%lld places, the first %lld: %lld\n", (long long)n, (long long)first, (long long)got);
        }
    const int64_t large[] = {8257, 65 * 64 + 1, 64 * 64 * 64, 64 * 64 * 64 + 1, 1048576, 1048577, ((int64_t)1 << 32) - 1};
    for (int64_t n : large)
        for (int64_t i = 0; i < 20000; ++i) {
            const int64_t first = i < 10000 ? n - 1 - i % n : (int64_t)((unsigned long long)i * 2654435761ull % (unsigned long long)n);
            const int64_t got = find(n, first, &rounds);
            if (rounds > most) most = rounds;
            if (got != first && bad++ < 20) printf("%lld places, the first %lld: %lld\n", (long long)n, (long long)first, (long long)got);
        }
    printf("%d wrong, %d rounds\n", bad, most);
    return bad != 0 || most > 7;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_every_place_is_found(tmp_path):
    src, exe = tmp_path / "probes.cpp", tmp_path / "probes"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    done = subprocess.run([str(exe)], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout
