"""Sizes at which the operators take the paths that small batches leave out. test_operator_shapes.py holds them against the rules that cut the work."""

# join: (rows, columns, types). A workgroup of either direction takes two turns or more, the last one of some of them only; a row has 16 to 1024 lanes, and rows
# of whole pieces of 8 columns and others take turns
JOIN_TURNS = [(33003, 24, "f32"), (33001, 100, "bf16"), (17005, 250, "mixed"), (9003, 500, "bf16"), (4611, 777, "f32"), (5003, 1024, "mixed"), (2561, 2048, "bf16"),
              (2307, 2051, "mixed"), (2111, 4096, "bf16"), (2103, 8000, "bf16"), (2090, 8191, "f32")]
