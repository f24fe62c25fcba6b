"""Sizes of products that together take every tile of every kind: (type, rows, cin, cout, behind an activation and dropout, elements by which the
tensors are off their alignment).  Most are a little beyond, or short of, whole tiles and slices."""

SIZES = [
    # 128 x 192 in all three products, and 128 x 128 for the weights' gradient
    ("bf16", 16330, 760, 2296, True, 0), ("bf16", 16330, 1144, 2296, True, 0),
    # large tiles, rows of whole 16 bytes, of odd values, of whole words
    ("bf16", 16400, 776, 2312, True, 0), ("bf16", 16400, 776, 2312, True, 1), ("bf16", 16400, 776, 2312, True, 2), ("bf16", 16384, 768, 2304, False, 0),
    ("bf16", 65552, 264, 72, True, 0), ("bf16", 65551, 265, 71, True, 0), ("bf16", 65552, 266, 74, False, 0),
    # narrow outputs
    ("bf16", 88055, 72, 9, False, 0), ("bf16", 88055, 73, 9, False, 0), ("bf16", 88055, 74, 10, False, 0),
    # many rows, small weights
    ("bf16", 40001, 136, 40, True, 0), ("bf16", 40001, 137, 41, True, 0), ("bf16", 40001, 138, 42, True, 0),
    # few rows, large weights
    ("bf16", 130, 1848, 4056, True, 0), ("bf16", 130, 1848, 4056, False, 1), ("bf16", 130, 1848, 4056, True, 2), ("bf16", 64, 2304, 768, False, 0),
    # fp32
    ("f32", 16400, 776, 2312, True, 0), ("f32", 16400, 775, 2309, True, 0), ("f32", 16390, 260, 772, False, 0), ("f32", 16390, 259, 771, True, 0),
    ("f32", 40001, 64, 72, True, 0), ("f32", 16384, 256, 768, False, 1), ("f32", 64, 2304, 768, True, 0), ("f32", 63, 2303, 767, True, 0),
]
