"""Batches of requests behind a shared prefix for which the bf16 attention takes each of its forms.

(form, pieces of the prefix, (query heads, KV heads, head dimension), [(requests, rows, own keys), ..], prefix, bytes of scratch
or None for what the library asks for)"""

LLAMA = (32, 8, 128)
SMALL = (8, 2, 128)
NARROW = (4, 2, 64)

FORMS = {
    "tokens, four wavefronts": ("TOKENS", 0, SMALL, [(1, 1, 65), (1, 3, 3), (1, 9, 130), (1, 1, 0)], 77, None),
    "tokens, two wavefronts": ("TOKENS", 0, LLAMA, [(40, 1, 33), (5, 9, 70), (1, 20, 20), (3, 2, 0)], 45, None),
    "tokens, two wavefronts, narrow": ("TOKENS", 0, NARROW, [(120, 1, 33), (9, 20, 70), (40, 3, 3)], 45, None),
    "rows": ("ROWS", 0, LLAMA, [(1, 150, 150), (1, 1, 1), (2, 77, 200), (1, 211, 211), (1, 40, 9), (1, 33, 0)], 45, None),
    "rows without a prefix": ("ROWS", 0, LLAMA, [(2, 150, 150), (1, 1, 1), (2, 77, 200), (1, 211, 211), (1, 40, 9)], 0, None),
    "rows behind whole tiles": ("ROWS", 0, LLAMA, [(3, 100, 128), (2, 128, 128), (1, 64, 64)], 128, None),
    "rows, narrow": ("ROWS", 0, NARROW, [(70, 150, 150), (20, 64, 200), (9, 77, 30)], 100, None),
    "tiles": ("TILES", 1, LLAMA, [(100, 8, 8), (20, 9, 0), (8, 3, 40)], 1027, None),
    "tiles, pieces": ("TILES", 32, LLAMA, [(5, 8, 8), (1, 13, 13)], 14000, None),
    "split": ("SPLIT", 3, SMALL, [(1, 1, 700)], 1500, None),
    "split, many rows": ("SPLIT", 20, SMALL, [(20, 1, 100), (1, 9, 1300), (3, 1, 0)], 5001, None),
    "split, own keys alone": ("SPLIT", 0, SMALL, [(1, 1, 3001), (1, 8, 2500), (1, 2, 9)], 0, None),
    "split, narrow": ("SPLIT", 20, NARROW, [(20, 1, 100), (1, 9, 1300)], 5001, None),
    "split, narrow, one row": ("SPLIT", 12, NARROW, [(1, 1, 100)], 3001, None),
    "tiles and split": ("TILES_SPLIT", 32, LLAMA, [(5, 8, 300), (1, 3, 1100)], 14000, None),
    "finish": ("TILES_FINISH", 6, LLAMA, [(125, 1, 20), (3, 1, 70)], 1500, None),
    "finish, four wavefronts": ("TILES_FINISH", 32, LLAMA, [(20, 1, 30), (2, 1, 0)], 14003, None),
    "no scratch": ("TOKENS", 0, SMALL, [(1, 1, 700), (1, 5, 5)], 1500, 0),
    "a little scratch": ("SPLIT", 1, SMALL, [(1, 1, 700)], 1500, 12500),
}

# float32: 128 rows a workgroup, for either head dimension
WIDE_F32 = {
    "128": (LLAMA, [(3, 150, 150), (6, 100, 130), (2, 1, 1), (4, 97, 40), (1, 64, 0)], 517),
    "128, no prefix": (LLAMA, [(7, 150, 150), (6, 100, 130), (2, 1, 1), (4, 97, 40), (1, 64, 0)], 0),
    "64": ((16, 4, 64), [(40, 150, 150), (6, 100, 130), (2, 1, 1), (12, 97, 40), (1, 64, 0)], 33),
}


def requests_of(spec):
    out, row, key = [], 0, 0
    for n, rows, own in spec:
        for _ in range(n):
            out.append((row, rows, key, own))
            row += rows + (rows == 3)                  # (now and then a row of nobody)
            key += (own + 7) // 8 * 8
    return out
