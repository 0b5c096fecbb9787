"""CPU: tokens are divided by the page size with a product and a shift; the constants hold for every page size and every token below 2^31."""
import random

from tests.helpers import host_program

PROGRAM = r"""
#include <cstdint>
#include <cstdio>
#include <cuda_runtime.h>
#include "step_ops.h"
int main() {
    long long n;
    int page;
    while (std::scanf("%lld %d", &n, &page) == 2) {
        unsigned magic, shift;
        dps::page_division(page, magic, shift);
        std::printf("%lld\n", (long long)(((uint64_t)(unsigned)n * magic) >> shift));
    }
}
"""


def test_division(tmp_path, monkeypatch):
    monkeypatch.setenv("CPLUS_INCLUDE_PATH", "/usr/local/cuda/include")
    run = host_program(tmp_path, PROGRAM)
    rng = random.Random(1)
    pages = [*range(1, 300), 2 ** 31 - 1, 2 ** 30, 2 ** 30 + 1, 2 ** 30 - 1, *(rng.randrange(1, 2 ** 31) for _ in range(500)), *(rng.randrange(1, 5000) for _ in range(500))]
    lines = []
    for d in pages:
        most = (2 ** 31 - 1) // d
        for q in {1, 2, most, max(most - 1, 1), rng.randint(1, most)}:
            lines += [(n, d) for n in (q * d - 1, q * d, min(q * d + d - 1, 2 ** 31 - 1)) if 0 <= n < 2 ** 31]
        lines += [(0, d), (2 ** 31 - 1, d)]
    for (n, d), (got,) in zip(lines, run(lines)):
        assert got == n // d, (n, d)
