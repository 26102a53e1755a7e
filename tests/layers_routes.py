"""Sizes that reach every kernel of the products, and the kernels that they are meant to reach: test_layers_routes asserts that the library chooses
those (without a device), test_gpu_layers_routes that their results are right."""

# T, rows, in, out, elements between rows, what is in the epilogue: "light" nothing, "full" activation, dropout, residual and the stored input -> kernel
FORWARD = []
for T in ("f32", "f16", "bf16", "f8"):
    FORWARD += [
        (T, 17, 64, 40, 0, "full", "few"),
        (T, 20001, 301, 257, 2, "full", "product 64") if T == "f32" else (T, 33333, 301, 47, 2, "full", "product 64"),
        (T, 45000, 133, 257, 3, "full", "product 128"),
        (T, 20000, 272, 264, 0, "full", "chunks"),
    ]
    if T in ("f16", "bf16"):
        FORWARD += [(T, 9000, 2056, 2064, 0, "full", "long"), (T, 9000, 1032, 2064, 0, "light", "long"), (T, 9000, 1032, 2064, 0, "full", "chunks")]
    else:
        FORWARD += [(T, 9000, 2064, 1032, 0, "light", "chunks")]

# T, type of dY, rows, in, out, elements between rows -> kernel of dA, kernel of dW, whether dW's sum is made in parts
BACKWARD = []
for T in ("f32", "f16", "bf16"):
    long = "chunks" if T == "f32" else "long"
    BACKWARD += [
        (T, T, 300, 33, 47, 1, "product 64", "product 64", True),
        (T, T, 45000, 133, 257, 3, "product 128", "product 128", True),
        (T, T, 200, 264, 136, 0, "chunks", "chunks", False),
        (T, T, 1000, 264, 136, 0, "chunks", "chunks", True),
        (T, T, 33000, 520, 264, 0, long, long, True),
        (T, T, 520, 4104, 4096, 0, "chunks", long, False),
    ]
    BACKWARD += [(T, O, 20000, 264, 264, 0, "chunks", long, True) for O in ("f32", "f16", "bf16") if O != T]
