"""Sizes of projections and gated blocks that reach each of the ways on which their products run, with ends inside a tile on every side
and k that is no multiple of a stage: (kind, rows, N, K, forward (tiles, in parts), backward (tiles, dx in parts, dw in parts)).
Which way a size takes is asserted without a GPU, the results on one."""
from paper_2606_02091_amd import dflare as dfl

T64, T128, HALVES, T256 = dfl.TILES_64, dfl.TILES_128, dfl.TILES_128_64, dfl.TILES_256
WAYS = [
    ("linear", 33, 72, 72, (T64, False), (T64, False, False)),
    ("linear", 65, 72, 72, (T128, False), (T128, False, False)),
    ("gated", 33, 72, 72, (T64, False), (T64, False, False)),
    ("gated", 129, 72, 72, (HALVES, False), (T128, False, False)),
    ("linear", 63, 1032, 2056, (T64, True), (T64, True, False)),
    ("linear", 48, 9728, 2560, (T64, True), (T64, True, False)),
    ("linear", 33, 264, 4104, (T64, True), (T64, False, False)),
    ("linear", 67, 712, 72, (T128, False), (T128, True, False)),
    ("linear", 129, 1160, 1032, (T128, True), (T128, True, False)),
    ("linear", 795, 1544, 72, (HALVES, False), (T128, True, True)),
    ("linear", 5511, 2232, 72, (T256, False), (T128, False, True)),
    ("linear", 135, 10952, 3256, (T256, True), (T256, True, False)),
    ("linear", 387, 136, 11544, (T128, True), (T256, False, False)),
    ("linear", 1025, 72, 5928, (T128, True), (T256, False, True)),
    ("linear", 5781, 2568, 664, (T256, False), (T256, True, True)),
    ("gated", 63, 520, 2056, (T64, True), (T64, True, False)),
    ("gated", 33, 72, 456, (T64, True), (T64, False, False)),
    ("gated", 300, 520, 2056, (T128, True), (T128, False, False)),
    ("gated", 729, 744, 72, (T128, False), (T128, True, True)),
    ("gated", 667, 9016, 72, (T256, False), (T128, True, False)),
    ("gated", 131, 8312, 2296, (T256, True), (T256, True, False)),
    ("gated", 201, 136, 11224, (T128, True), (T256, False, False)),
    ("gated", 1551, 72, 3336, (T128, True), (T256, False, True)),
    ("gated", 5821, 1304, 680, (T256, False), (T256, True, True)),
]
