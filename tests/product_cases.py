"""Products of 8-bit operands, (dtype, m, k, n), by the kernel that each is for: every kernel of every type, with one block of columns, two, three, four
and more, odd and even numbers of them, a last block that is partly there, rows and outputs that end inside a tile, fewer and more tiles than workgroups."""
FEW16, FEW32, FEW64 = "rowwise_f8_few_kernel<{}, 1, 2, 8>", "rowwise_f8_few_kernel<{}, 2, 2, 8>", "rowwise_f8_few_kernel<{}, 2, 4, 4>"
GROUPS, MIDDLE, LARGE = "rowwise_f8_kernel<{}, 64, 128, 1, 2, 2>", "rowwise_f8_kernel<{}, 128, 128, 2, 2, 1>", "rowwise_f8_kernel<{}, 256, 256, 4, 2, 1>"

# (outputs a multiple of 8 come out as vectors where they are aligned, others by way of LDS in the large tiles)
CASES = {
    FEW16: [("bf16", 3, 2064, 200), ("f32", 3, 2064, 200), ("bf16", 5, 400, 41), ("f32", 5, 400, 41)],
    FEW32: [("bf16", 20, 128, 200), ("f32", 20, 128, 200), ("bf16", 65, 256, 41), ("f32", 65, 256, 41)],
    FEW64: [("bf16", 100, 400, 5000), ("f32", 100, 400, 5000), ("bf16", 150, 144, 3000), ("f32", 130, 656, 4097), ("f32", 61, 2064, 8200)],
    GROUPS: [("bf16", 61, 2064, 8200), ("bf16", 513, 528, 2049), ("bf16", 300, 1040, 3904), ("bf16", 515, 656, 3304), ("f32", 515, 656, 3304), ("f32", 5000, 400, 257), ("f32", 515, 1040, 3303)],
    MIDDLE: [("bf16", 6000, 16, 392), ("f32", 6000, 16, 392), ("bf16", 2000, 128, 2056), ("f32", 1999, 144, 2500), ("bf16", 2049, 384, 4104), ("f32", 520, 1040, 4096), ("bf16", 1030, 528, 2051),
             ("f32", 1850, 656, 7117)],
    LARGE: [("bf16", 7999, 16, 9992), ("bf16", 7999, 128, 9991), ("bf16", 3999, 144, 11992), ("bf16", 3999, 256, 11991), ("bf16", 2499, 272, 11992), ("bf16", 2500, 384, 11991),
            ("bf16", 2499, 400, 11992), ("bf16", 2500, 512, 11992), ("bf16", 2499, 528, 11992), ("bf16", 2400, 1040, 11992), ("bf16", 2400, 640, 11991), ("bf16", 2499, 656, 4992),
            ("bf16", 2499, 1040, 4999)],
}
FLAT = [(kernel, *c) for kernel, cases in CASES.items() for c in cases]
