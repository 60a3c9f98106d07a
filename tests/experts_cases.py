"""Sizes at which products grouped by expert take each of their ways: rows of each expert, rows behind the last one's, outs, ins, the type, and the ways
of the products, of the rows' gradient and of the weights'.  A way is a cut of experts_cut.h, whether sums are made in parts and, of tiles
of 256, whether there are whole rounds, and how what is left behind them goes."""
SHORT = [500, 20, 0, 350, 130, 77, 256, 200, 30, 10, 90, 300] * 2
LONG = [800, 620, 0, 350, 630, 77, 856, 500, 300, 110, 390, 900] * 2

CASES = [
    ([2000, 100, 0, 1800, 300], 5, 4104, 264, "bf16", "WIDE rounds quarters", "FEW128 parts", "ANY128"),
    ([2000, 100, 0, 1800, 300], 5, 264, 4104, "bf16", "FEW128 parts", "WIDE rounds quarters", "ANY128"),
    (LONG, 9, 1544, 72, "bf16", "WIDE rounds tiles", "FEW128 parts", "ANY128"),
    (LONG, 9, 72, 1544, "bf16", "FEW128 parts", "WIDE rounds tiles", "ANY128"),
    (SHORT, 9, 1544, 72, "bf16", "WIDE tiles", "RING128 parts", "WIDE tiles"),
    (SHORT, 9, 72, 1544, "bf16", "RING128 parts", "WIDE tiles", "WIDE tiles"),
    ([1024, 0, 512, 767, 511, 1280], 0, 4096, 136, "bf16", "WIDE rounds", "FEW128 parts", "WIDE quarters"),
    ([1024, 0, 512, 767, 511, 1280], 0, 136, 4096, "bf16", "FEW128 parts", "WIDE rounds", "WIDE quarters"),
    ([512, 0, 256, 768, 511], 0, 4096, 264, "bf16", "WIDE quarters", "FEW128 parts", "WIDE tiles"),
    ([512, 0, 256, 768, 511], 0, 264, 4096, "bf16", "FEW128 parts", "WIDE quarters", "WIDE tiles"),
    ([3900, 3, 0, 4300], 1, 1992, 136, "bf16", "WIDE rounds small", "FEW128 parts", "WIDE quarters"),
    ([3900, 3, 0, 4300], 1, 136, 1992, "bf16", "FEW128 parts", "WIDE rounds small", "WIDE quarters"),
    ([1300, 0, 2100, 700], 3, 1032, 264, "bf16", "FEW128", "RING128", "WIDE quarters"),
    ([1300, 0, 2100, 700], 3, 264, 1032, "bf16", "RING128", "FEW128", "WIDE quarters"),
    ([150, 0, 200, 130, 160], 0, 2056, 2056, "bf16", "RING128 parts", "RING128 parts", "WIDE rounds tiles"),
    ([200, 41, 0, 305], 2, 4104, 1032, "bf16", "RING128", "RING128 parts", "WIDE rounds quarters"),
    ([250, 0, 140, 155], 0, 2048, 2048, "bf16", "FEW128 parts", "FEW128 parts", "WIDE rounds"),
    ([30, 0, 9], 2, 584, 40, "bf16", "RING32", "RING32 parts", "ANY128"),
    ([30, 0, 9], 2, 40, 584, "bf16", "RING32 parts", "RING32", "ANY128"),
    ([3000, 0, 905], 7, 128, 264, "bf16", "RING32", "RING32", "ANY128 parts"),
    ([i % 4 for i in range(1100)], 3, 64, 72, "bf16", "ANY32", "ANY32", "ANY128"),
    ([1125, 2040, 0, 5420], 4, 43, 396, "bf16", "ANY64 parts", "ANY32", "ANY128 parts"),
    ([1125, 2040, 0, 5420], 4, 396, 43, "bf16", "ANY32", "ANY64 parts", "ANY128 parts"),
    (LONG, 5, 42, 598, "bf16", "ANY64 parts", "ANY64", "ANY128"),
    (LONG, 5, 598, 42, "bf16", "ANY64", "ANY64 parts", "ANY128"),
    (LONG[:12], 3, 43, 2895, "bf16", "ANY128 parts", "ANY64", "ANY128"),
    (LONG[:12], 3, 2895, 43, "bf16", "ANY64", "ANY128 parts", "ANY128"),
    ([1975, 5378, 0, 9838], 2, 521, 43, "bf16", "ANY128", "ANY128 parts", "ANY128 parts"),
    ([1975, 5378, 0, 9838], 2, 43, 521, "bf16", "ANY128 parts", "ANY128", "ANY128 parts"),
    ([90, 0, 32], 2, 355, 41, "bf16", "ANY32", "ANY32 parts", "ANY128"),
    ([90, 0, 32], 2, 41, 355, "bf16", "ANY32 parts", "ANY32", "ANY128"),
    ([1125, 2040, 0, 5420], 4, 43, 396, "f32", "ANY64 parts", "ANY64", "ANY128 parts"),
    ([1125, 2040, 0, 5420], 4, 396, 43, "f32", "ANY64", "ANY64 parts", "ANY128 parts"),
    (LONG, 5, 42, 598, "f32", "ANY32 parts", "ANY128", "ANY128 parts"),
    (LONG, 5, 598, 42, "f32", "ANY128", "ANY32 parts", "ANY128 parts"),
    ([1975, 5378, 0, 9838], 2, 521, 43, "f32", "ANY128", "ANY128 parts", "ANY128 parts"),
    ([1975, 5378, 0, 9838], 2, 43, 521, "f32", "ANY128 parts", "ANY128", "ANY128 parts"),
    ([90, 0, 32], 2, 41, 53, "f32", "ANY32", "ANY32", "ANY128"),
    ([600, 0, 1500], 1, 264, 136, "f32", "ANY32", "ANY32 parts", "ANY128 parts"),
]

_ROWS = {cut + parts for cut in ("RING32", "RING128", "FEW128") for parts in ("", " parts")}
_ANY = {cut + parts for cut in ("ANY32", "ANY64", "ANY128") for parts in ("", " parts")}
_WIDE = {"WIDE rounds", "WIDE tiles", "WIDE quarters", "WIDE rounds tiles", "WIDE rounds quarters"}
_SUMS = {"ANY128", "ANY128 parts"}

# What CASES have to reach, by product, type and whether memory can fill tiles directly.
WAYS = {(kind, "bf16", True): _ROWS | _WIDE | {"WIDE rounds small"} for kind in (0, 1)}
WAYS.update({(kind, dtype, False): _ANY for kind in (0, 1) for dtype in ("bf16", "f32")})
WAYS.update({(2, "bf16", True): _WIDE | _SUMS, (2, "bf16", False): _SUMS, (2, "f32", False): _SUMS})


def direct(counts, outs, ins, dtype):
    """Whether memory can fill tiles directly, of contiguous tensors."""
    return dtype == "bf16" and outs % 8 == 0 and ins % 8 == 0 and len(counts) <= 1024


def tiles(kind, counts, outs, ins):
    """Tiles of 256 that a call has."""
    def cut(n):
        return -(-n // 256)
    return len(counts) * cut(outs) * cut(ins) if kind == 2 else sum(map(cut, counts)) * cut(ins if kind else outs)
