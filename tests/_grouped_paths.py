"""Which kernel a product by kind of row takes, and how often its sums are rounded.

The rules are those of grouped_kernels.hpp, written down again so that a test can say which loops it is meant for."""
from tests._products import EPS

SIZE = {"f32": 4, "f64": 8}
TILE = {"f32": 128, "f64": 64}      # lines of a full tile, and columns of a tile of gW


def near(rows, ld, prec):
    return rows * ld < 2 ** 31 // SIZE[prec]


def reached(rows, comps, perm):
    """Rows that a descriptor has to span."""
    return rows if perm else min(rows, 1024 // comps + 2)


def lines_of_products(rows, terms, n, comps, perm, ld_from, ld_to, matrix, prec):
    """("stream", lines a workgroup), ("rows", lines a tile) or ("far", lines a tile)."""
    lines = rows * comps
    if terms <= 128 and near(reached(rows, comps, perm), max(ld_from, ld_to), prec):
        wide = 128 if prec == "f32" and n > 64 else 64
        shift = 10
        while shift > 6 and (lines >> shift) * -(-n // wide) < 1024:
            shift -= 1
        return "stream", 1 << shift
    if not near(reached(rows, comps, perm), ld_from, prec) or not near(matrix, 1, prec):
        return "far", TILE[prec]
    return "rows", TILE[prec] // 2 if lines // TILE[prec] * -(-n // 64) < 512 else TILE[prec]


def positions_of_a_chunk(rows, k, n, comps, prec):
    tiles, shift = -(-k // 64) * -(-n // TILE[prec]), 20
    least = max(256, 4 * k * n // (k + n))
    while shift > 4 and (((rows >> shift) * tiles < 1600 and comps << (shift - 1) >= least) or ((rows >> shift) * tiles < 320 and comps << (shift - 1) >= 64)):
        shift -= 1
    return 1 << shift


def up(v):
    return (v + 255) // 256 * 256


def workspace(rows, k, n, comps, prec):
    chunks = -(-rows // positions_of_a_chunk(rows, k, n, comps, prec))
    slots = 2 * chunks if chunks > 1 else 0
    return up(slots * k * n * SIZE[prec]) + up(slots * n * 8)


def chain(terms, prec):
    """Roundings one after another in a sum of products.  fp32: an instruction adds 32 products of parts to its sums, six of them make 32 terms; each may round (or cut,
    which is two half steps) the sums once, and inside it 32 products of its own; what the parts leave out is one more.  fp64: every term rounds once."""
    steps = -(-terms // 32)
    return 2 * (6 * steps + 34) if prec == "f32" else 32 * steps


def tolerances(ref, rows, k, n, comps, most, prec):
    """most: positions of the largest group.  gW: a chunk's chain, then its chunks one after another; out has its bias."""
    chunk = positions_of_a_chunk(rows, k, n, comps, prec)
    joins = -(-most // chunk) + 9
    counts = {"out": chain(k, prec) + 2, "gx": chain(n, prec), "gW": chain(min(most, chunk) * comps, prec) + joins}
    tiny = 1e-37 if prec == "f32" else 1e-300
    return {name: EPS[prec] * c * ref[name][1] + tiny for name, c in counts.items()}
