"""Sizes of linear_int8 by the kernel that they take: (kernel, (m, n, k), alignment of the 8-bit rows).

Kernels: "rows F J" of few rows (F times 16 rows and J times 16 columns a workgroup; "by XCD" where its workgroups are dealt to
the XCDs by rows), "tile 128", "tile 256" and "halves" (tiles of 128 in halves), "split" where their reduction is."""

KERNELS = [
    ("rows 1 1", (1, 10, 4096), 16), ("rows 1 1", (3, 70, 4500), 4), ("rows 1 1", (16, 33, 9001), 1), ("rows 1 1", (2, 40, 8400), 16),
    ("rows 1 1 by XCD", (130, 10, 48), 16), ("rows 1 1 by XCD", (131, 20, 20), 4), ("rows 1 1 by XCD", (130, 10, 17), 1),
    ("rows 1 2", (1, 10, 16), 16), ("rows 1 2", (3, 70, 36), 4), ("rows 2 2", (50, 2050, 16), 16), ("rows 2 2", (50, 2050, 20), 4),
    ("rows 1 2", (51, 2050, 19), 1), ("rows 1 2", (7, 4170, 1001), 1),
    ("rows 2 1", (131, 515, 1024), 16), ("rows 2 1", (200, 515, 1004), 4), ("rows 2 1", (200, 515, 1011), 1),
    ("rows 2 1 by XCD", (2051, 20, 1024), 16), ("rows 2 1 by XCD", (1030, 100, 140), 4), ("rows 2 1 by XCD", (2051, 20, 301), 1),
    ("rows 1 2", (100, 2050, 16), 16), ("rows 1 2", (100, 2050, 20), 4), ("rows 2 2", (203, 515, 19), 1),
    ("rows 4 1", (300, 515, 272), 16), ("rows 4 1", (257, 515, 300), 4), ("rows 4 1", (257, 515, 301), 1),
    ("rows 4 1 by XCD", (700, 300, 16), 16), ("rows 4 1 by XCD", (700, 300, 20), 4), ("rows 4 1 by XCD", (700, 515, 19), 1),
    ("rows 4 2", (300, 4100, 48), 16), ("rows 4 2", (50, 4170, 300), 4), ("rows 4 2", (131, 2050, 19), 1),
    ("tile 128", (2051, 2050, 48), 16), ("tile 128", (2051, 2050, 140), 4), ("tile 128", (2050, 2050, 301), 1),
    ("tile 256", (2050, 4100, 272), 16), ("tile 256", (2051, 4099, 1001), 1),
    ("halves", (500, 2050, 16), 16), ("halves", (777, 1365, 1001), 1), ("halves", (700, 2050, 300), 4),
    ("halves split", (1, 10, 20000), 16), ("halves split", (5, 33, 20001), 1),
    ("tile 128 split", (20, 4100, 20000), 16), ("tile 256 split", (130, 8200, 20000), 16),
]


def name(case):
    return f"{case[0]}: {case[1][0]}x{case[1][1]}x{case[1][2]}"


def copied(case):
    """Bytes of x and w that tiles have copied: rows that do not start at multiples of 16 bytes, or of x end inside of some."""
    m, n, k = case[1]
    return 0 if case[2] == 16 else (m + n) * k


def kernel(choice, m, n):
    """The name of what (variant, splits, row_blocks, row_columns) launches."""
    variant, splits, blocks, columns = choice
    if variant == 3:
        return f"rows {blocks} {columns}" + (" by XCD" if -(-m // (16 * blocks)) >= 8 else "")
    return {0: "tile 128", 1: "tile 256", 2: "halves"}[variant] + (" split" if splits > 1 else "")
