"""Which variant of the selection kernel an eviction gets: CTAs to a row, threads to a CTA."""
from tests import host_rules

# rows, room of a row; CTAs to a row, threads
TABLE = [
    (1, 16, 1, 256), (64, 1024, 1, 256), (64, 1025, 1, 1024), (65, 2048, 1, 256), (65, 2049, 1, 1024), (1, 2048, 1, 1024),
    (1, 4095, 1, 1024), (1, 4096, 2, 1024), (1, 8191, 2, 1024), (1, 8192, 4, 1024), (1, 16383, 4, 1024), (1, 16384, 8, 1024),
    (8, 1 << 20, 8, 1024), (9, 1 << 20, 4, 1024), (16, 65536, 4, 1024), (16, 8191, 2, 1024), (17, 65536, 2, 1024), (32, 65536, 2, 1024),
    (33, 65536, 1, 1024), (1 << 26, 1 << 30, 1, 1024), (1, 1 << 30, 8, 1024),
]


def test_the_rule():
    for field, column in (("ranks", 2), ("threads", 3)):
        got = host_rules.evaluate("cache_choice.h", f"sparsed::choose_evict_variant(rows, static_cast<int>(room)).{field}", "rows room",
                                  [row[:2] for row in TABLE])
        assert got == [row[column] for row in TABLE]
