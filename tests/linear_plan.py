"""Which kernel a product of the linear operator takes, worked out from the constants of
flashlinear.hip's plan, and sizes that take each of them.

A kernel is written as its letter and tile: s256 (streamed, 256 x 256 tiles), e128 (streamed,
with rows that end inside a vector of 8), c64 (checked); with "/" behind it where the
reduction axis is split and "+" where a workgroup takes more than one tile, so that the ring
runs on over their border."""
import os
import re

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_10071_amd", "csrc",
                   "flashlinear.hip")
CUS = 256


def _costs(src, name):
    body = re.search(name + r"\[\] = \{(.*?)\};", src, re.S)[1]
    rows = re.findall(r"\{(\d+), (?:(\d+) \* )?kCus, ([\d.]+)f, ([\d.]+)f\}", body)
    return [(int(t), int(r or 1) * CUS, float(step), float(fixed)) for t, r, step, fixed in rows]


def costs():
    src = open(SRC).read()
    return {n: _costs(src, n) for n in ("kStream16", "kStream32", "kChecked")}


def up(a, b):
    return -(-a // b)


def plan(table, rows, cols, red, es):
    """(tile, parts, workgroups at once) with the least estimated time."""
    total, best = up(red, 128 // es), None
    for tile, resident, step, fixed in table:
        tiles, split = up(rows, tile) * up(cols, tile), 1
        while split == 1 or (split <= total // 2 and split * tiles <= 2 * resident):
            steps = up(total, split)
            parts = up(total, steps)
            us = up(tiles * parts, resident) * (fixed + step * steps)
            if parts > 1:
                us += 3 + parts * rows * cols * 2e-6
            if best is None or us < best[0]:
                best = (us, tile, parts, resident)
            split *= 2
    return best[1:]


def kernel(tables, rows, cols, red, es, along_a, along_b, padded=False):
    """The kernel of C = A B^T over `red` elements of rows at 16-byte places."""
    e = 16 // es
    whole = (padded or (red if along_a else rows) % e == 0) and (red % e if along_b else cols % 8) == 0
    table = tables["kChecked" if not whole else "kStream32" if es == 4 else "kStream16"]
    tile, parts, resident = plan(table, rows, cols, red, es)
    more = whole and up(rows, tile) * up(cols, tile) * parts > resident
    return (f"{('e' if along_b and cols % 8 else 's') if whole else 'c'}{tile}"
            + "/" * (parts > 1) + "+" * more)


def kernels(tables, M, K, N, es, formed=False):
    """The kernels of the forward, the input's and the weight's gradient, for more than 32
    rows; `formed`: with an activation or another type of output."""
    padded = formed or (N % 8 != 0 and K % 8 == 0)
    return (kernel(tables, M, N, K, es, True, True), kernel(tables, M, K, N, es, True, False, padded),
            kernel(tables, N, K, M, es, False, False, padded))


# (M, K, N), and the forward's kernel for 16-bit and for float32 inputs
FORWARD = [
    ((40001, 40, 200), "s256", "s256"), ((40001, 40, 203), "e256", "e256"),
    ((6000, 200, 2056), "s256", "s256"), ((6000, 200, 2059), "e256", "e256"),
    ((12000, 200, 2056), "s256+", "s256+"), ((12000, 200, 2059), "e256+", "e256+"),
    ((9001, 104, 2056), "s128+", "s128+"), ((9001, 104, 2059), "e128+", "e128+"),
    ((20000, 72, 72), "s128", "s64+"), ((20000, 72, 75), "e128", "e64+"),
    ((20000, 2056, 72), "s128/", "s64+"), ((20000, 2056, 75), "e128/", "e64+"),
    ((9001, 1032, 72), "s64", "s128/"), ((9001, 1032, 75), "e64", "e128/"),
    ((40001, 129, 72), "c128", "c128"), ((40001, 129, 75), "c128", "c128"),
]

# (M, K, N), and the kernels of the input's and the weight's gradient, for both
BACKWARD = [
    ((12000, 136, 72), ("s128", "s64/"), ("s64+", "s64/")),
    ((40001, 264, 72), ("s128+", "s128/"), ("s128+", "s64/")),
    ((200, 2056, 4099), ("s128/", "s256"), ("s128/", "s64+")),
    ((200, 2056, 2056), ("s64/", "s128"), ("s128/", "s64+")),
    ((40001, 520, 72), ("s256+", "s128/"), ("s256+", "s64/")),
    ((9001, 1032, 72), ("s256", "s64/"), ("s256", "s64/")),
    ((9001, 515, 72), ("c128", "c64/"), ("c128", "c64/")),
    ((3500, 2056, 72), ("s128", "s64/"), ("s128", "s128/")),
    ((40001, 2056, 200), ("s256+", "s256/"), ("s128+", "s256/")),
]
