"""Calls over windows with sinks and over trees that go to the kernel for many (row, head) columns: test_host_launches_spans.py checks
that they do, test_gpu_spans_wide.py their answers."""
from paper_2501_05408_amd import tempo as T

BF16, E4M3 = T.TEMPO_BF16, T.TEMPO_E4M3

WIDE = [  # store, what, Hq, Hkv, D, Z, B, t, rows, window, sinks, steps of their own, rows of their own
    (BF16, "prompt", 128, 2, 128, 32, 8, 520, 30, 4, 4, False, False),          # windows shorter than a group, far from their sinks
    (BF16, "prompt", 24, 8, 128, 32, 16, 1, 180, 12, 100, False, True),         # sinks of four groups that reach into the rows
    (BF16, "prompt", 8, 2, 128, 256, 2, 764, 176, 2150, 40, False, False),      # split
    (BF16, "prompt", 24, 8, 64, 32, 4, 371, 1000, 349, 40, False, True),         # many tiles of columns, runs of them to a die
    (BF16, "prompt", 128, 2, 64, 32, 8, 1563, 54, 33, 4, False, False),
    (BF16, "prompt", 24, 8, 64, 256, 3, 5030, 35, 3050, 40, False, False),      # ten splits
    (E4M3, "prompt", 64, 4, 128, 256, 16, 9, 120, 50, 4, False, True),
    (E4M3, "prompt", 32, 8, 128, 32, 16, 103, 66, 4, 100, False, False),        # 96 columns
    (E4M3, "prompt", 64, 4, 128, 64, 1, 7336, 185, 2924, 100, False, False),    # split; the first window lies more than 64 tiles from the sinks
    (E4M3, "prompt", 128, 1, 64, 256, 8, 73, 74, 1836, 100, False, False),
    (E4M3, "prompt", 16, 4, 64, 32, 3, 3049, 700, 3771, 0, False, True),        # split
    (BF16, "block", 128, 8, 128, 32, 16, 4516, 18, 21, 4, False, False),        # 96 columns, a window more than 64 tiles from the sinks
    (BF16, "block", 128, 1, 64, 32, 16, 7249, 38, 3, 4, False, False),          # the same, heads of 64
    (BF16, "block", 6, 2, 128, 32, 16, 4149, 226, 1924, 40, True, False),       # one range of more than 64 tiles
    (BF16, "block", 8, 8, 128, 256, 8, 2274, 33, 3712, 40, False, False),       # 64 columns: two wavefronts without any
    (BF16, "block", 12, 4, 128, 32, 8, 974, 24, 948, 100, False, False),        # 96 columns, split
    (E4M3, "block", 128, 8, 128, 32, 16, 3943, 29, 2, 4, False, False),
    (E4M3, "block", 24, 8, 128, 32, 4, 5267, 233, 2273, 0, True, False),        # one range of more than 64 tiles
    (E4M3, "block", 8, 1, 64, 32, 16, 2026, 201, 2418, 4, False, False),        # the same, heads of 64
    (E4M3, "block", 64, 8, 64, 32, 16, 5179, 20, 3505, 100, False, False),      # 96 columns, split, far sinks
    (BF16, "tree", 8, 8, 128, 32, 1, 3547, 68, 0, 0, False, False),             # more than 64 nodes; 96 columns, 23 splits
    (BF16, "tree", 64, 4, 64, 32, 2, 2180, 235, 0, 0, False, False),            # one range of more than 64 tiles
    (BF16, "tree", 24, 8, 128, 64, 16, 1, 81, 198, 100, True, False),
    (BF16, "tree", 4, 1, 128, 64, 16, 1351, 27, 1098, 0, True, False),          # window, split
    (BF16, "tree", 128, 1, 128, 32, 16, 4033, 15, 1, 40, False, False),         # a node sees the sinks and itself
    (BF16, "tree", 128, 8, 128, 32, 4, 4881, 3, 0, 0, False, False),            # 64 columns
    (E4M3, "tree", 64, 2, 128, 32, 16, 8, 64, 0, 0, False, False),
    (E4M3, "tree", 64, 1, 64, 32, 4, 2978, 173, 5, 100, False, False),
    (E4M3, "tree", 64, 4, 64, 32, 2, 1974, 222, 0, 0, False, False),            # one range of more than 64 tiles
    (E4M3, "tree", 128, 8, 128, 32, 4, 417, 71, 9, 4, True, False),
    (E4M3, "tree", 64, 1, 128, 32, 2, 4755, 49, 0, 0, True, False),             # split
    (BF16, "tree", 24, 8, 64, 32, 16, 700, 200, 0, 0, True, True),
    (E4M3, "tree", 128, 8, 128, 32, 4, 417, 140, 9, 4, True, True),
    (E4M3, "tree", 64, 4, 128, 32, 2, 1500, 250, 700, 33, False, False),        # the bits of 250 nodes beside the codes
]
