"""Lists that take one launch, a cluster of CTAs per worker, with odd sizes: up to 16 pieces of 2048 elements (all calls) and up to
64 (all but the Adam step)."""

SIXTEEN = [1, 7, 0, 8, 9, 63, 64, 65, 255, 1000, 2047, 2048, 2049, 4096 + 17]
SIXTY_FOUR = [98_305] + SIXTEEN[1:]
# sizes, types, n, shift (as tensor_lists.make takes them)
LISTS = [
    (sizes, types, n, shift) for sizes in (SIXTEEN, SIXTY_FOUR)
    for types, n, shift in ((["f32"], 1, 1), (["bf16"], 2, 4), (["f16"], 1, 2), (["f32", "bf16", "f16"], 3, 0), (["f16", "f32", "bf16", "bf16"], 2, 5),
                            (["bf16", "f32"], 64 if sizes is SIXTEEN else 7, 3))
] + [([2049, 33], ["f32", "bf16"], 1, 7), ([1023, 1025], ["f16"], 2, 1), ([3], ["f16"], 1, 6)]


def pieces(sizes):
    return sum(-(-s // 2048) for s in sizes)
