"""Sizes of the linear weight gradient by the kernels that they take: (rows, n, k) of a bf16 dY, and the launches."""

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
