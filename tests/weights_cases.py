"""Prompts whose entry weights two stretches of keys a block gather, with more row
tiles than the waves of a block have on their way at once.  Test infrastructure
only."""
import torch

BF, F32 = torch.bfloat16, torch.float32

TWO_STRETCHES = [
    # dtype, D, Hq, Hkv, page, lengths, rows, how rows see: "last", "rising", "any"
    (BF, 128, 16, 8, 16, [471, 300, 512, 64, 449, 385, 130, 1], 333, "last"),
    (BF, 128, 16, 8, 16, [471, 63, 511, 0, 448, 320, 131, 33], 297, "any"),
    (BF, 128, 16, 8, 64, [465, 65, 200, 512, 448, 511, 100, 2], 520, "rising"),
    # one, two and more stretches of a sequence, odd and even, none
    (BF, 128, 8, 8, 16, [130, 64, 65, 0, 192, 193, 256, 255, 1, 70, 120], 600, "any"),
    # more row tiles than are looked through at once
    (BF, 64, 64, 8, 16, [500, 449, 66, 0, 512, 300, 1, 129], 1030, "any"),
    (BF, 64, 64, 8, 8, [512, 449, 385, 64, 130, 300, 201, 129], 1027, "last"),
    (F32, 128, 16, 8, 16, [250, 32, 33, 0, 97, 256, 160, 1], 150, "last"),
    (F32, 128, 32, 8, 32, [256, 224, 31, 128, 64, 255, 100, 7], 77, "any"),
    (F32, 64, 16, 8, 16, [470, 512, 64, 65, 1, 0, 300, 129], 290, "rising"),
    (F32, 64, 64, 32, 16, [250, 1, 128], 300, "any"),
]


def row_tiles(case):
    """Tiles of 16 rows (query, head of the group) of a (sequence, KV head)."""
    return -(-case[6] * (case[2] // case[3]) // 16)


def requested_ahead(case):
    """Row tiles that the eight waves of a block have on their way."""
    return 8 * (2 if case[1] * (2 if case[0] == BF else 4) > 256 else 4)
