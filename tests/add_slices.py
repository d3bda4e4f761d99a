"""Sizes for every way in which workgroups share a tile's reduction in the product with a residual, and what tells on the host that they still take that way."""
import paper_2305_13525_amd as axo

COUNTERS = 8192  # bytes ahead of the sums in a workspace of axo_fc_add
FEW = ((16, 32), (32, 32), (16, 64), (16, 128))  # rows x columns of the tiles whose waves split the reduction
WHOLE = (128, 128)

# (rows, columns of the tiles) -> tokens x in-features x out-features.  Of 128 x 128 tiles two to sixteen slices, the last of them shorter or not, edges inside a tile and on it, rows of X that
# start on cache lines and that do not
SLICED = [((16, 32), (1, 2219, 8)), ((16, 32), (33, 8192, 200)), ((32, 32), (1, 6130, 1020)), ((16, 64), (1, 9416, 933)), ((16, 128), (1, 13373, 3797)),
          (WHOLE, (70, 4127, 11458)), (WHOLE, (42, 7728, 6995)), (WHOLE, (256, 8192, 1536)), (WHOLE, (4118, 5147, 9)), (WHOLE, (2184, 6899, 73)), (WHOLE, (707, 6246, 270)),
          (WHOLE, (129, 6000, 1025)), (WHOLE, (640, 4096, 256)), (WHOLE, (300, 8192, 520)), (WHOLE, (287, 9235, 745)), (WHOLE, (300, 8192, 512))]


def up(a, b):
    return -(-a // b)


def sliced_on(m, k, n):
    """The (rows, columns, slices) that the size of the workspace can stand for."""
    size, steps, found = axo.axo_fc_add_workspace_bytes(axo.Problem.make((1, 1, 1), (0, 0, 0), m, k, n)), up(k, 64), set()
    for rows, cols in FEW + (WHOLE,):
        tiles = up(m, rows) * up(n, cols)
        if size <= COUNTERS or (size - COUNTERS) % (tiles * rows * cols * 4):
            continue
        slices = (size - COUNTERS) // (tiles * rows * cols * 4)
        # of equal numbers of steps, but for the last; those of few rows a whole number of sixteen steps or so, as many as CUs leave room for
        asked = [max(1, min(256 // tiles, steps // 16, 16))] if (rows, cols) != WHOLE else range(2, 17)
        if slices > 1 and any(up(steps, up(steps, a)) == slices for a in asked):
            found.add((rows, cols, slices))
    return found
