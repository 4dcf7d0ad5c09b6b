"""Sizes at which the products take each of their large tiles, with the plan that the rules of gsq_plan.h must
choose there: test_products_plan.py pins the plans on the host, test_gpu_product_tiles.py runs the cases.  So a
rule that changes cannot leave a kernel without its test in silence."""

L2, L3, L4 = (-0.5, 0.5), (-1.0, 0.0, 1.0), (-1.5, -0.5, 0.5, 1.5)
L8, L16 = tuple(k - 3.5 for k in range(8)), tuple(k - 7.5 for k in range(16))

# y ("forward"), dx ("input_grad") and the 8-bit y ("int8"): rows of each group, O, I, elements that the arrays begin
# past an aligned address, plan (whole workgroups "ring" or shared sums "split", height x width)
ROWS = [
    ("forward", [4000], 8200, 520, 0, "ring 256x256"),
    ("forward", [900, 30, 0, 200, 370, 77], 8200, 136, 0, "ring 256x256"),
    ("forward", [1000], 4104, 1032, 0, "ring 128x256"),
    ("forward", [1000], 4000, 264, 0, "ring 64x256"),
    ("forward", [4100], 2050, 515, 0, "ring 128x128"),
    ("forward", [3000, 0, 2900, 70], 2051, 1003, 1, "ring 128x128"),
    ("input_grad", [4000], 520, 8200, 0, "ring 256x256"),
    ("input_grad", [900, 30, 0, 200, 370, 77], 136, 8200, 0, "ring 256x256"),
    ("input_grad", [1000], 1032, 4104, 0, "ring 128x256"),
    ("input_grad", [1000], 264, 4000, 0, "ring 64x256"),
    ("input_grad", [4100], 4099, 4001, 0, "ring 128x128"),
    ("input_grad", [3000, 0, 2900, 70], 1001, 8001, 0, "ring 128x128"),
    ("input_grad", [6000], 2048, 4096, 3, "ring 128x128"),
    ("int8", [3000], 8200, 528, 0, "ring 256x256"),
    ("int8", [900, 30, 0, 200, 370, 77], 8200, 272, 0, "ring 256x256"),
    ("int8", [4000], 8201, 112, 0, "ring 256x256"),        # one slab, which ends early
    ("int8", [1000], 4100, 272, 0, "ring 128x256"),
    ("int8", [700], 5000, 400, 0, "ring 64x256"),
    ("int8", [4100], 2050, 1029, 0, "ring 128x128"),
    ("int8", [3000, 0, 2900, 70], 2051, 1040, 5, "ring 128x128"),
]

# dW ("weight_grad") and H ("gram"): as above, of H the O is not used
SUMS = [
    ("weight_grad", [4100], 8200, 8200, 0, "ring 256"),
    ("weight_grad", [9000, 40, 0, 9100], 4104, 2056, 0, "ring 256"),
    ("weight_grad", [600, 0, 33], 2056, 4104, 0, "ring 128"),
    ("weight_grad", [600, 0, 33], 2051, 4097, 0, "ring 128"),
    ("gram", [12000], 0, 8200, 0, "ring 256"),
    ("gram", [9000, 70, 0, 9100], 0, 4104, 0, "ring 256"),
    ("gram", [600, 0, 33], 0, 4104, 0, "ring 128"),
    ("gram", [600, 0, 33], 0, 4101, 0, "ring 128"),
]

# the packed layer: layout, levels, group size, rows of each group, O, I, elements past an aligned address, plan
PACKED = [
    ("group", L2, 128, [2100], 8200, 1280, 0, "ring 256x256"),
    ("group", L2, 16, [2100], 8200, 48, 0, "ring 256x256"),
    ("group", L3, 64, [1100], 4100, 1088, 0, "ring 128x256"),
    ("group", L4, 64, [1000], 4079, 64, 0, "ring 64x256"),
    ("group", L4, 16, [1000], 4079, 560, 0, "ring 64x256"),
    ("base3", L3, 32, [900, 30, 0, 200, 370, 77], 8200, 160, 0, "ring 256x256"),
    ("base3", L3, 256, [700], 6001, 1024, 0, "ring 128x256"),
    ("group", L8, 128, [900, 30, 0, 200, 370, 77], 8200, 384, 0, "ring 256x256"),
    ("group", L8, 32, [1100], 4100, 1056, 0, "ring 128x256"),
    ("group", L8, 64, [1000], 4079, 576, 0, "ring 64x256"),
    ("group", L8, 16, [900, 30, 0, 200, 370, 77], 8200, 208, 0, "ring 256x256"),
    ("superblock", L8, 16, [900, 30, 0, 200, 370, 77], 8200, 256, 0, "ring 256x256"),
    ("superblock", L8, 16, [1100], 4100, 1280, 0, "ring 128x256"),
    ("superblock", L4, 16, [1000], 4080, 512, 0, "ring 64x256"),
    ("group", L16, 64, [2100], 8200, 320, 0, "ring 256x256"),
    ("group", L16, 16, [900, 30, 0, 200, 370, 77], 8200, 176, 0, "ring 256x256"),
    ("group", L16, 128, [1100], 4100, 1152, 0, "ring 128x256"),
    ("group", L16, 256, [1000], 4090, 768, 0, "ring 64x256"),
    # x from an odd address
    ("group", L2, 128, [1100], 4100, 1280, 1, "ring 128x256"),
    ("group", L2, 16, [2100], 8201, 48, 1, "ring 128x256"),
    ("base3", L3, 64, [900, 30, 0, 200, 370, 77], 4104, 320, 3, "ring 128x256"),
    ("group", L4, 16, [700], 4100, 560, 1, "ring 128x256"),
    ("group", L8, 64, [900, 30, 0, 200, 370, 77], 4104, 576, 7, "ring 128x256"),
    ("superblock", L8, 16, [900, 30, 0, 200, 370, 77], 4104, 256, 1, "ring 128x256"),
    ("group", L16, 64, [1100], 4100, 64, 1, "ring 128x256"),
    ("group", L16, 16, [700], 4111, 176, 2, "ring 128x256"),
    ("group", L8, 128, [70, 40, 0, 5, 17], 520, 640, 1, "split 16x16"),
    ("superblock", L8, 16, [8] * 64, 72, 256, 1, "split 16x16"),   # experts, eight tokens each
    ("superblock", L8, 16, [32] * 64, 2048, 256, 1, "ring 128x256"),
]


def tight(kind, o, i, shift):
    """Whether all operands' rows are aligned to 16 bytes."""
    unit = 16 if kind == "int8" else 8
    return shift == 0 and i % unit == 0 and (kind in ("forward", "int8") or o % unit == 0 or kind == "gram")


def label(case):
    return "-".join(str(len(v)) if isinstance(v, tuple) else str(v).replace(" ", "") for v in case)
