"""Sizes of the linear weight gradient by the kernels that they take: (rows, n, k) of a bf16 dY, and the launches."""

# whole groups of 16 bytes, in tiles of 256: steps of 32 tokens that end with 8, 1, 31 and 32, whole and in parts
ALIGNED = [
    ((200, 4096, 4096), ["big"]),
    ((513, 2568, 4096), ["big"]),
    ((2079, 4096, 2304), ["big"]),
    ((4097, 2048, 3008), ["big", "join_kernelILj1ELj2E"]),
    ((8192, 1288, 2304), ["big", "join_kernelILj1ELj4E"]),
    ((16385, 1024, 1024), ["big", "join_kernelILj1ELj8E"]),
]

# tiles of 128, of either type: from one token and one column on
SMALL = [
    ((1, 1, 1), ["wgrad_kernel"]), ((1, 8, 16), ["wgrad_kernel"]), ((2, 9, 17), ["wgrad_kernel"]),
    ((15, 200, 208), ["wgrad_kernel"]), ((17, 130, 140), ["wgrad_kernel"]), ((33, 257, 130), ["wgrad_kernel"]),
    ((63, 7, 300), ["wgrad_kernel"]), ((95, 300, 15), ["wgrad_kernel"]),
    ((1000, 40, 1030), ["wgrad_kernel", "join"]), ((4099, 129, 257), ["wgrad_kernel", "join"]),
]

RAGGED = [
    # whole sums; the last token behind 6 whole steps and 7 tokens, behind 16 whole steps, and behind 64
    ((200, 4091, 4095), ["big"]),
    ((513, 2565, 4095), ["big"]),
    ((2049, 4091, 2300), ["big"]),
    # in 2, 3, 4, 6 and 41 parts; the whole tiles of 17 columns of them beside the parts of the others
    ((4097, 2041, 3007), ["big", "join_kernelILj1ELj2E"]),
    ((4110, 2565, 1790), ["big", "join_kernelILj1ELj4E"]),
    ((8200, 1285, 2300), ["big", "join_kernelILj1ELj4E"]),
    ((8200, 1023, 2300), ["big", "join_kernelILj1ELj8E"]),
    ((65500, 1285, 249), ["big", "join_kernelILj8ELj4E"]),
    ((4096, 4095, 4097), ["big", "join_kernelILj1ELj8E"]),
]
