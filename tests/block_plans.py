"""Sizes of the products over row groups by the tiles they take: every kind in every product, whole and in parts."""

# rows, hidden, ffn, group_off (None: one group), activation, and the plan of each product
FFN = [
    (1, 64, 64, None, "silu", dict(up=("few8", 1), down=("few8", 1), dh=("wide", 1), dx=("small", 1), dw=("small", 1))),
    (5, 64, 8192, None, "gelu", dict(up=("few8", 1), down=("few8", 16), dh=("wide", 1), dx=("small", 16), dw=("small", 1))),
    (5, 8256, 64, None, "silu", dict(up=("few8", 16), down=("few8", 1), dh=("small", 16), dx=("small", 1), dw=("small", 1))),
    (300, 2048, 4096, None, "silu", dict(up=("small", 2), down=("small", 8), dh=("small", 4), dx=("small", 8), dw=("small", 1))),
    (290, 4096, 2112, None, "gelu", dict(up=("small", 4), down=("small", 4), dh=("small", 8), dx=("small", 4), dw=("small", 1))),
    (3001, 64, 64, [0, 1, 2987], "silu", dict(up=("few8", 1), down=("few8", 1), dh=("wide", 1), dx=("small", 1), dw=("small", 16))),
    (8190, 64, 64, [7, 4000, 4033, 8190], "silu",
     dict(up=("few4", 1), down=("few4", 1), dh=("wide", 1), dx=("small", 1), dw=("small", 16))),
    (2100, 4096, 64, None, "silu", dict(up=("small", 16), down=("wide", 1), dh=("small", 16), dx=("small", 1), dw=("small", 4))),
    (2100, 64, 4096, None, "gelu", dict(up=("small", 1), down=("small", 16), dh=("wide", 1), dx=("small", 8), dw=("small", 2))),
    # the weights' gradients of wide tiles: groups of one partial stage, of whole ones, of many, and empty ones
    (2100, 4096, 192, [3, 40, 40, 168, 1001, 1002, 2097], "silu",
     dict(up=("small", 8), down=("wide", 1), dh=("small", 8), dx=("wide", 1), dw=("wide", 1))),
    (12000, 1024, 1024, [3, 40, 7041, 11990], "silu",
     dict(up=("wide", 1), down=("wide", 1), dh=("wide", 1), dx=("wide", 1), dw=("wide", 1))),
    (8190, 512, 1408, [0, 64, 5000, 8190], "gelu",
     dict(up=("wide", 1), down=("small", 1), dh=("wide", 1), dx=("wide", 1), dw=("wide", 1))),
    # a training step's experts, fine-grained experts, and a dense block
    (4531, 2048, 1408, [0, 700, 1290, 1290, 1291, 1700, 1764, 1990, 2300, 2565, 2600, 2983, 3300, 3520, 4000, 4031, 4531], "silu",
     dict(up=("small", 1), down=("wide", 1), dh=("small", 1), dx=("wide", 1), dw=("wide", 1))),
    (16384, 2048, 768, [0, 5286] + [5286 + 358 * i + i % 7 for i in range(1, 31)] + [16384], "silu",
     dict(up=("wide", 1), down=("wide", 1), dh=("wide", 1), dx=("wide", 1), dw=("wide", 1))),
    (8192, 4096, 14336, None, "silu",
     dict(up=("wide", 1), down=("wide", 1), dh=("wide", 1), dx=("wide", 1), dw=("wide", 1))),
]

# rows, depth, channels, group_off, activation, plan
I8 = [
    (1, 448, 48, None, "none", ("few8", 1)),
    (1, 4160, 48, None, "none", ("few8", 16)),
    (5, 28736, 144, None, "silu", ("few8", 16)),
    (31, 1408, 2064, None, "gelu", ("few8", 1)),
    (8190, 448, 48, [7, 4000, 4033, 8190], "none", ("few4", 1)),
    (8190, 448, 48, [0, 33, 4000, 8188], "silu", ("few4", 1)),
    (12000, 576, 144, None, "none", ("small", 1)),
    (12000, 448, 272, None, "silu", ("small", 1)),
    (2100, 8256, 48, None, "none", ("small", 16)),
    (2100, 8256, 48, None, "silu", ("small", 16)),
    # wide tiles: four stages whose last is a half, and whole ones
    (6007, 448, 528, None, "none", ("wide", 1)),
    (8190, 448, 1040, [5, 2500, 2501, 8188], "silu", ("wide", 1)),
    # a long prefill's down projection, and its gate and up; ragged experts, one token
    (16384, 14336, 4096, None, "none", ("wide", 1)),
    (8192, 4160, 28672, None, "silu", ("wide", 1)),
    (6007, 2048, 2816, [0, 1200, 1957, 2500, 2500, 2900, 3301, 3600, 3900, 4160, 4416, 4650, 4900, 5200, 5460, 5761, 6007], "silu",
     ("small", 1)),
    (1, 4096, 28672, None, "silu", ("few8", 1)),
]


def groups(off):
    return 1 if off is None else len(off) - 1
