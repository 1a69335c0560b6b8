"""Sizes of moe_ffn by the kernels that they take: {kind of weights: [(kernels, (rows, f, d, experts, top_k))]}.

Kinds: "f32"; "16", weights of f16 or bf16; "int8", whatever the type of x.  Kernels: how rows are routed ("logits": in a launch of
their own; "routing": by every workgroup of the up projections), the up projections (4 columns a wavefront, or 16, 32 or 64 rows of
an expert at a time; how many wavefronts share a reduction; "parts": several workgroups share an expert's columns), and the down
projection (4 columns, by workgroups of 8 or 16 wavefronts; 32 columns; or by experts, 16 or 32 rows at a time, with so many
wavefronts to a reduction; "split" where workgroups share its rows and columns; "few rows" where a workgroup has less than it can)."""
import ctypes


class Choice(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in (
        "up_variant", "down_variant", "up_blocks", "up_waves", "up_parts", "fused", "apart", "down_waves", "down_parts",
        "down_blocks", "down_rows", "splits", "chunk")]


def names(c, top_k):
    """(routing, up, down): the names of what is launched"""
    routing = ", ".join(["logits"] * c.apart + ["routing" if c.fused else "route"])
    up = ("4 columns", "16 rows", f"{16 * c.up_blocks} rows")[c.up_variant] + f", {c.up_waves} share" + ", parts" * (c.up_parts > 1)
    if c.down_variant == 2:
        return routing, up, f"by experts, {16 * c.down_blocks} rows, {c.down_waves} share" + ", parts" * (c.down_parts > 1)
    down = f"4 columns, {c.down_waves} wavefronts" if c.down_variant == 0 else "32 columns"
    return routing, up, down + ", split" * (c.splits > 1) + ", few rows" * (c.down_rows < min(64, 512 // top_k))



KERNELS = {
    "f32": [
        ("routing | 4 columns, 1 share | 4 columns, 16 wavefronts", (1, 18, 19, 1, 1)),
        ("logits, routing | 4 columns, 2 share | 4 columns, 16 wavefronts, split", (2, 62, 339, 17, 8)),
        ("route | 4 columns, 8 share | 4 columns, 8 wavefronts", (3, 31, 1251, 12, 4)),
        ("logits, route | 4 columns, 4 share | 4 columns, 16 wavefronts", (4, 23, 658, 65, 2)),
        ("routing | 16 rows, 8 share | 32 columns", (10, 20, 17, 1, 1)),
        ("logits, routing | 16 rows, 8 share | 32 columns, split", (10, 20, 19, 18, 1)),
        ("route | 32 rows, 8 share, parts | 32 columns, few rows", (37, 18, 17, 1, 1)),
        ("logits, route | 32 rows, 8 share | 32 columns, split, few rows", (67, 17, 18, 17, 4)),
        ("logits, route | 16 rows, 1 share | by experts, 16 rows, 2 share", (68, 170, 39, 166, 1)),
        ("logits, route | 16 rows, 1 share | by experts, 16 rows, 8 share", (85, 696, 17, 97, 1)),
        ("logits, route | 16 rows, 4 share | by experts, 16 rows, 1 share", (89, 18, 511, 146, 2)),
        ("logits, route | 16 rows, 1 share | by experts, 16 rows, 4 share", (98, 326, 21, 162, 1)),
        ("logits, route | 32 rows, 1 share, parts | 32 columns, split, few rows", (137, 65, 18, 65, 16)),
        ("logits, route | 16 rows, 1 share | 32 columns, split", (141, 17, 17, 155, 1)),
        ("route | 32 rows, 4 share | by experts, 16 rows, 8 share, parts", (176, 708, 471, 12, 1)),
        ("route | 32 rows, 4 share, parts | 32 columns, split", (275, 25, 302, 128, 16)),
        ("route | 32 rows, 2 share | by experts, 16 rows, 2 share, parts", (296, 152, 148, 55, 3)),
        ("route | 16 rows, 2 share | by experts, 16 rows, 1 share, parts", (400, 52, 179, 198, 1)),
        ("route | 32 rows, 2 share, parts | 32 columns, split", (951, 36, 129, 106, 4)),
        ("route | 32 rows, 1 share | by experts, 16 rows, 4 share, parts", (1167, 340, 39, 80, 2)),
    ],
    "16": [
        ("routing | 4 columns, 1 share | 4 columns, 16 wavefronts", (1, 18, 19, 1, 1)),
        ("logits, routing | 4 columns, 2 share | 4 columns, 16 wavefronts, split", (2, 62, 339, 17, 8)),
        ("route | 4 columns, 8 share | 4 columns, 8 wavefronts", (4, 20, 1198, 5, 5)),
        ("logits, route | 4 columns, 4 share | 4 columns, 16 wavefronts", (4, 41, 675, 162, 4)),
        ("logits, routing | 16 rows, 4 share | 4 columns, 16 wavefronts, split", (8, 199, 373, 31, 4)),
        ("routing | 16 rows, 8 share | 32 columns", (10, 20, 17, 1, 1)),
        ("route | 64 rows, 8 share, parts | 32 columns, few rows", (37, 18, 17, 1, 1)),
        ("logits, route | 32 rows, 8 share | 32 columns, split, few rows", (67, 17, 18, 17, 4)),
        ("logits, route | 16 rows, 8 share | by experts, 16 rows, 1 share", (68, 41, 196, 282, 1)),
        ("logits, route | 16 rows, 1 share | by experts, 16 rows, 8 share", (72, 529, 26, 155, 1)),
        ("logits, route | 16 rows, 1 share | by experts, 16 rows, 2 share", (78, 203, 36, 297, 1)),
        ("logits, route | 32 rows, 2 share | by experts, 32 rows, 1 share", (85, 123, 179, 97, 16)),
        ("logits, route | 16 rows, 1 share | by experts, 16 rows, 2 share, parts", (85, 134, 109, 145, 2)),
        ("logits, route | 16 rows, 1 share | by experts, 16 rows, 4 share", (96, 427, 23, 224, 1)),
        ("route | 64 rows, 8 share | by experts, 32 rows, 2 share, parts", (97, 173, 1113, 14, 8)),
        ("logits, route | 16 rows, 1 share | by experts, 16 rows, 4 share, parts", (111, 394, 27, 199, 2)),
        ("logits, route | 64 rows, 1 share, parts | 32 columns, split, few rows", (137, 65, 18, 65, 16)),
        ("logits, route | 16 rows, 1 share | 32 columns, split", (141, 17, 17, 155, 1)),
        ("logits, route | 32 rows, 4 share | by experts, 32 rows, 2 share", (171, 198, 461, 23, 2)),
        ("logits, route | 64 rows, 4 share | by experts, 32 rows, 8 share, parts", (204, 626, 300, 21, 3)),
        ("logits, route | 16 rows, 1 share | by experts, 16 rows, 8 share, parts", (222, 613, 18, 197, 1)),
        ("route | 64 rows, 4 share, parts | 32 columns, split", (275, 25, 302, 128, 16)),
        ("route | 32 rows, 2 share | by experts, 32 rows, 4 share, parts", (280, 437, 151, 32, 2)),
        ("route | 16 rows, 2 share | by experts, 16 rows, 1 share, parts", (351, 74, 132, 242, 1)),
        ("route | 32 rows, 1 share | by experts, 32 rows, 4 share", (558, 381, 36, 153, 4)),
        ("route | 32 rows, 1 share | by experts, 32 rows, 8 share", (581, 1461, 18, 80, 2)),
        ("route | 64 rows, 2 share | by experts, 32 rows, 1 share, parts", (893, 93, 179, 128, 4)),
        ("route | 64 rows, 2 share, parts | 32 columns, split", (951, 36, 129, 106, 4)),
        ("route | 64 rows, 1 share | 32 columns, split", (1136, 20, 19, 130, 3)),
    ],
    "int8": [
        ("routing | 4 columns, 1 share | 4 columns, 16 wavefronts", (1, 18, 19, 1, 1)),
        ("logits, routing | 4 columns, 2 share | 4 columns, 16 wavefronts", (2, 40, 590, 20, 4)),
        ("route | 4 columns, 4 share | 4 columns, 8 wavefronts", (3, 18, 1072, 6, 2)),
        ("logits, route | 4 columns, 8 share | 32 columns", (3, 22, 2650, 181, 1)),
        ("logits, routing | 16 rows, 2 share | 4 columns, 16 wavefronts, split", (6, 110, 293, 38, 16)),
        ("route | 16 rows, 4 share | 32 columns, split", (6, 1607, 567, 6, 1)),
        ("routing | 16 rows, 8 share | 32 columns", (10, 20, 17, 1, 1)),
        ("route | 32 rows, 8 share, parts | 32 columns, few rows", (37, 18, 17, 1, 1)),
        ("route | 32 rows, 4 share, parts | 32 columns, split, few rows", (43, 2039, 529, 2, 2)),
        ("logits, route | 32 rows, 8 share | 32 columns, split, few rows", (67, 17, 18, 17, 4)),
        ("logits, route | 32 rows, 1 share, parts | 32 columns, split, few rows", (137, 65, 18, 65, 16)),
        ("logits, route | 16 rows, 1 share | 32 columns, split", (141, 17, 17, 155, 1)),
        ("logits, route | 32 rows, 1 share | 32 columns, split, few rows", (162, 33, 20, 89, 8)),
        ("route | 32 rows, 4 share | 32 columns, split", (268, 17, 542, 149, 8)),
        ("route | 32 rows, 2 share, parts | 32 columns, split", (275, 25, 302, 128, 16)),
        ("route | 32 rows, 2 share | 32 columns, split", (294, 18, 261, 156, 8)),
    ],
}


def cases(kind):
    return [size for _, size in KERNELS[kind]]
