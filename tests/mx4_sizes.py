"""Sizes of MXFP4 products that reach each kernel of the tiles, and how: test_mx4_choice.py
says that they do, test_gpu_mx4_tiles.py runs them.

(kernel, M, N, K): 256 CUs.  Per kernel whole and cut tiles, rows of y that begin at half
cache lines (N % 32 == 0: the stores past the caches) and that do not, an odd and an even
number of stages of 256 k; and, where it is ever taken for more tiles than there is room
for, work-groups that go on to a next tile."""

# room on 256 CUs
SLOTS = {"64x64": 256, "64x64 parts": 256, "64x128": 512, "64x128 parts": 256, "128x128": 512, "128x192": 256, "192x192": 256,
         "192x256": 256, "256x256": 256}
GATED_SLOTS = {"64x128": 256, "128x128": 512, "192x256": 256, "256x256": 256}

LINEAR = [
    ("64x64", 1060, 96, 288), ("64x64", 1026, 67, 32),
    ("64x64 parts", 1030, 96, 3040), ("64x64 parts", 1105, 73, 3808),
    ("64x128", 70, 8352, 320), ("64x128", 67, 8333, 32),
    ("64x128 parts", 200, 4128, 1312), ("64x128 parts", 75, 8210, 3104),
    ("128x128", 770, 13152, 448), ("128x128", 773, 13169, 32),
    ("128x192", 258, 13088, 864), ("128x192", 8336, 396, 1248),
    ("192x192", 779, 9376, 1056), ("192x192", 7602, 1033, 800), ("192x192", 1176, 13408, 1120), ("192x192", 8878, 1795, 896),
    ("192x256", 1045, 14656, 288), ("192x256", 1164, 13170, 32),
    ("256x256", 2338, 10304, 864), ("256x256", 1820, 13098, 544), ("256x256", 2182, 11040, 576)]

GATED = [
    ("64x128", 1060, 96, 288), ("64x128", 1026, 35, 32),
    ("128x128", 386, 11328, 352), ("128x128", 385, 11011, 32),
    ("192x256", 642, 11168, 800), ("192x256", 540, 13230, 544),
    ("256x256", 908, 14912, 288), ("256x256", 785, 14036, 608)]

# (N a multiple of 32)
QUANTIZED = [
    ("64x128", 1060, 96, 288), ("64x128", 1026, 32, 32),
    ("128x128", 386, 11328, 352), ("128x128", 387, 10976, 32),
    ("192x256", 642, 11168, 800), ("192x256", 540, 13248, 544),
    ("256x256", 908, 14912, 288), ("256x256", 785, 14048, 608)]


def tile(kernel, gated):
    """Rows and outputs of a tile."""
    rows, weight = (int(n) for n in kernel.split()[0].split("x"))
    return rows, weight // 2 if gated else weight


def tiles(kernel, gated, M, N):
    rows, outputs = tile(kernel, gated)
    return -(-M // rows) * -(-N // outputs)
