"""Sizes at which the operators take the paths that small batches leave out. test_operator_shapes.py holds them against the rules that cut the work."""

# join: (rows, columns, types). A workgroup of either direction takes two turns or more, the last one of some of them only; a row has 16 to 1024 lanes, and rows
# of whole pieces of 8 columns and others take turns
JOIN_TURNS = [(33003, 24, "f32"), (33001, 100, "bf16"), (17005, 250, "mixed"), (9003, 500, "bf16"), (4611, 777, "f32"), (5003, 1024, "mixed"), (2561, 2048, "bf16"),
              (2307, 2051, "mixed"), (2111, 4096, "bf16"), (2103, 8000, "bf16"), (2090, 8191, "f32")]

# weight gradient from a checkpoint: rows, in, out, type of dy, accumulate, elements behind a row of dy and of the gradient, in front of the first;
# then what the rule makes of it: large tiles, ranges, and values per thread of the launch that adds them (0: none)
WEIGHT_GRADS = [(517, 4090, 4090, "bfloat16", False, 0, 0, True, 1, 0), (513, 4096, 4096, "bfloat16", True, 8, 0, True, 1, 0),
                (6000, 2050, 2056, "bfloat16", True, 3, 1, True, 3, 4), (3001, 2050, 2056, "bfloat16", False, 0, 0, True, 3, 4),
                (12001, 1530, 1500, "bfloat16", False, 5, 2, True, 7, 1), (1001, 4090, 2041, "float32", False, 3, 1, True, 1, 0),
                (517, 4090, 4090, "float32", True, 0, 0, True, 1, 0), (3001, 2050, 2056, "float32", True, 0, 0, True, 3, 4),
                (9000, 2300, 1900, "float32", False, 4, 3, True, 5, 4), (16300, 1020, 1015, "float32", False, 1, 0, True, 8, 1),
                (16300, 1020, 1015, "bfloat16", True, 0, 0, False, 4, 1), (515, 4090, 4100, "bfloat16", False, 1, 1, False, 1, 0)]
