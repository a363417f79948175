"""Which kernel a packed attention call goes to, on a device of any size: the rule's own arithmetic, compiled for the host."""
import os
import subprocess

import pytest

from paper_2509_24014_b200 import build

# sequences, queries, keys in all, packed heads, tokens per tile, causal; whether it is the CTA-pair kernel
TABLE = [
    (0, 0, 0, 32, 128, 0, 0), (1, 1, 1, 32, 128, 1, 0),
    (8, 8 * 2048, 8 * 2048, 32, 128, 0, 0),                       # short: as fast on either
    (4, 4 * 4096, 4 * 4096, 32, 128, 0, 1), (1, 16384, 16384, 32, 128, 0, 1),
    (2, 2 * 8192, 2 * 8192, 32, 128, 1, 0), (1, 12288, 12288, 32, 128, 1, 1), (1, 32768, 32768, 32, 128, 1, 1),
    (1, 8192, 8192, 2, 128, 0, 0), (1, 8192, 8192, 3, 128, 0, 1),   # 32 and 48 clusters
    (1, 32768, 32768, 1, 128, 1, 0), (1, 32768, 32768, 2, 128, 1, 1),
    (3, 17000, 17000, 4, 18, 1, 1),                               # grouped heads: the diagonal costs less
    (4, 4 * 2048, 4 * 10240, 8, 32, 1, 1),                        # text that continues cached text
    (64, 64, 64 * 20000, 32, 128, 1, 0), (64, 64 * 500, 64 * 20000, 32, 128, 0, 0),   # few queries to a sequence
    (4, 16700, 16700, 32, 128, 1, 0),
]


def test_the_rule(tmp_path):
    main = tmp_path / "main.cc"
    main.write_text('#include <cstdio>\n#include "dense_choice.h"\nint main() { long long n, q, k; int h, t, c; '
                    'while (std::scanf("%lld %lld %lld %d %d %d", &n, &q, &k, &h, &t, &c) == 6) '
                    'std::printf("%d\\n", sparsed::packed_pair_pays(n, q, k, h, t, c != 0) ? 1 : 0); }\n')
    exe = tmp_path / "main"
    subprocess.run(["g++", "-std=c++17", "-I", build.CSRC, str(main), "-o", str(exe)], check=True)
    lines = "".join(" ".join(map(str, row[:6])) + "\n" for row in TABLE)
    out = subprocess.run([str(exe)], input=lines, capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in out] == [row[6] for row in TABLE]
