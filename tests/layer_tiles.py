"""Sizes whose products go through tiles of 256 x 256, in one pass over the GPU but for the last of FORWARD, with few and
with many steps of r.  (m, k, n, pad, type): pad is the columns by which the operands' rows are wider, 3 where they do not
start at 16-byte addresses, 5 where odd rows do."""
FORWARD = [(3500, 1000, 4075, 8, "bf16"), (3841, 72, 3841, 0, "fp16"), (3500, 1003, 4075, 3, "fp16"),
           (3300, 136, 3400, 8, "bf16"), (1500, 8200, 3000, 0, "bf16"), (1500, 8199, 3001, 3, "fp16"),
           (8200, 1000, 8100, 8, "bf16")]
EIGHT = [(3500, 2064, 4075, 16, "e4m3"), (3841, 1999, 3841, 3, "e4m3"), (3300, 144, 3400, 0, "e4m3"),
         (3000, 16400, 1500, 0, "e4m3")]
# dx [m, k] = dz w with sums over n, dw [n, k] = dz^T x with sums over m
DX = [(3500, 4072, 1000, 8, "bf16"), (3500, 4075, 1003, 5, "bf16"), (3841, 3848, 136, 0, "fp16"),
      (3500, 4075, 1003, 3, "fp16"), (1500, 3000, 8200, 0, "bf16")]
DW = [(1000, 4072, 3504, 8, "bf16"), (1000, 4075, 3507, 5, "bf16"), (136, 3848, 3848, 0, "fp16"),
      (1003, 4075, 3501, 3, "fp16"), (8200, 3000, 1500, 0, "bf16")]
SPLIT = [(1500, 8200, 3000), (1500, 8199, 3001), (3000, 16400, 1500), (1500, 3000, 8200), (8200, 3000, 1500)]


def products():
    """(rows, columns, length of the sums, bytes of an element, whether the sums are shared out) of every product."""
    for cases, pick in ((FORWARD, lambda m, k, n: (m, n, k)), (EIGHT, lambda m, k, n: (m, n, k)), (DX, lambda m, k, n: (m, k, n)),
                        (DW, lambda m, k, n: (n, k, m))):
        for m, k, n, _, kind in cases:
            yield (*pick(m, k, n), 1 if kind == "e4m3" else 2, (m, k, n) in SPLIT)
