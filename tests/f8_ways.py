"""Sizes (tokens, inputs, outputs) of products on 8-bit floats, by the way that a call of them takes."""
import ctypes

#: by rows, (tokens, outputs) of a workgroup in 16s
ROWS = {(1, 1): [(1, 304, 271), (1, 281, 334)], (1, 2): [(4, 256, 9000), (35, 257, 2418)],
        (2, 1): [(90, 384, 2000), (18, 329, 1161)], (4, 1): [(500, 1100, 500), (33, 291, 2200)]}
#: on tiles, (outputs, tokens, whether the reduction is split); the last ones of a list are no whole blocks
TILES = {(128, 64, False): [(1100, 640, 1531), (157, 384, 3000), (759, 246, 1054)],
         (128, 64, True): [(64, 9216, 4096), (16, 16384, 200), (459, 2171, 1467)],
         (128, 128, False): [(2305, 384, 776), (2200, 1100, 2100)],
         (128, 128, True): [(1652, 6528, 159), (491, 2226, 958)],
         (256, 128, False): [(3000, 640, 2100), (2403, 384, 1673)],
         (256, 128, True): [(2860, 8832, 162), (768, 19968, 3018)]}

ON_ROWS = [size for sizes in ROWS.values() for size in sizes]
ON_TILES = [size for sizes in TILES.values() for size in sizes]


class Way(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int) for name in ("rows", "tokens", "outs", "tile_outs", "tile_tokens", "parts", "run")]


def way(cnn, n, i, o):
    """The built-in choice (fc_f8_way)."""
    choose = cnn.lib._ZN3cnn9fc_f8_wayEiii
    choose.restype = Way
    return choose(n, i, o)
