"""Which tile a product takes, by the rules of csrc/int8.hip and csrc/mx8.hip with the constants that stand there: so that
a test of a tile notices when retuned constants send its sizes elsewhere.  Only tests import this module."""
import ast
import math
import os
import re

import torch

CSRC = os.path.join(os.path.dirname(__file__), "..", "paper_2601_01473_amd", "csrc")


def _source(name):
    with open(os.path.join(CSRC, name)) as f:
        return f.read()


def _tiles(text):
    table = re.search(r"static const Tile kTiles\[\] = (\{.*?\});", text, re.S).group(1)
    return ast.literal_eval(table.replace("{", "[").replace("}", "]"))


def _number(text, name):
    expression = re.search(r"constexpr int64_t %s = ([^;]+);" % name, text).group(1)
    return eval(expression.replace("(int64_t)", ""), {"__builtins__": {}})


def _up(a, b):
    return -(-a // b)


def int8(M, N, K):
    """(rows of a tile, parts of K); rows 0: the kernel of few rows."""
    text = _source("int8.hip")
    full, part_steps, near, few, few_rows, work = (
        _number(text, n) for n in ("kFullGrid", "kPartSteps", "kNear", "kFewTile", "kFewRows", "kFewWork"))
    if M <= few or (M <= few_rows and K <= work and M * K * _up(N, 16 * full) <= work and _up(N, 16) <= (1 << 23) - 8):
        return 0, 1
    steps = _up(_up(K, 16), 4)
    best = None
    for rows, step_near, step_far, step_full, ends in _tiles(text):
        tiles = _up(M, rows) * _up(N, rows)
        if tiles > (1 << 23) - 8:
            continue
        for grid in (1, 256, 512, 1024):
            parts = 1 if rows > 64 else max(1, min(grid // tiles, steps // part_steps))
            each, groups = math.ceil(steps / parts), tiles * parts / full
            busy = 0.0 if groups < 0.75 else (math.ceil(groups) if rows == 256 else groups) * each * step_full
            us = ends + max(each * (step_near if (M + N) * K <= near else step_far), busy)
            if parts > 1:
                us += 6 + parts * M * N * 8 / 3e6
            if best is None or us < best[0]:
                best = us, rows, parts
    return best[1:]


def weight_grad(g, K):
    """(way, rows and columns of a tile, parts of the rows) for a gradient g [M, N]; the way: "direct" (straight to LDS),
    "cut" (into planes first) or "registers"."""
    text = _source("mx8.hip")
    M, N = g.shape
    planes = {torch.float32: 3, torch.float16: 2, torch.bfloat16: 1}[g.dtype]
    if planes == 1 and g.data_ptr() % 16 == 0 and g.stride(0) % 8 == 0 and N % 8 == 0 and g.stride(0) >= N:
        way = "direct"
    else:
        way = "cut" if M * N >= 1 << 21 or (K >= 1024 and M >= 256) else "registers"
    part_steps, steps = _number(text, "kPartSteps"), _up(M, 32)
    best = None
    for rows, cols, alone, full, ends in _tiles(text):
        if full[planes - 1] == 0 or (rows > 64 and way == "registers"):
            continue
        tiles = _up(N, rows) * _up(K, cols)
        for grid in (1, 256, 512, 1024):
            parts = max(1, min(grid // max(1, tiles), steps // part_steps))
            each = _up(steps, parts)
            us = ends + max(each * alone[planes - 1], math.ceil(tiles * parts / 256) * each * full[planes - 1])
            if parts > 1:
                us += 6 + parts * N * K * 8 / 4e6
            if best is None or us < best[0]:
                best = us, rows, cols, parts
    return (way,) + best[1:]
