"""Sizes that take every variant of the attention kernels: (sequences, queries and keys of
each, heads, heads that share k and v, causal).  tests/test_attn_plan.py checks on the
CPU that they do; tests/test_gpu_attn_variants.py runs them."""

SHAPES = {
    "short": (40, 70, 70, 4, 1, True),          # whole, four waves; shared tiles of short keys
    "shared": (6, 40, 700, 4, 2, False),        # queries of two heads in a tile, split
    "single": (2, 1, 3000, 4, 2, True),         # split many times
    "medium": (1, 1300, 1300, 2, 1, True),      # everything split
    "dense": (2, 1000, 1000, 128, 1, True),       # whole, eight waves where there are
    "wide": (1, 1024, 8192, 16, 1, False),      # split, eight waves where there are
    "few keys": (1, 900, 40, 2, 2, False),      # keys' tiles split over the queries
}
WIDTHS = {64: 64, 96: 80, 128: 128, 256: 160}   # width of a kernel: a head of it
