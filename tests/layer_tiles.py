"""Sizes of the gated feed-forward block whose products of 16-bit types go to tiles of 256 x 256, more of them than compute units where nothing else is said:
(rows, dim, hidden), and what is expected of the products named: (tiles and pieces, at least; pieces along k; steps of 64 bytes along k, of one of the products of a sum, odd or not)."""
SEQUENCES = [
    ((3000, 136, 3400), {"gated": (257, 1, 1)}),                   # several tiles to a workgroup, an odd number of steps
    ((3000, 1001, 3400), {"gated": (257, 1, 0)}),                  # copies of operands, rows and columns that end inside a tile
    ((130, 3001, 3403), {"dw": (257, 1, 1)}),                      # a row for each k of both operands; the last step is filled up
    ((1203, 3000, 3400), {"dw": (257, 1, 0)}),
    ((6001, 4100, 264), {"dx": (257, 1, 1)}),                      # a sum of two products
    ((1200, 4500, 4500), {"dx": (257, 5, 1), "dw": (257, 1, 0)}),  # pieces along k, several to a workgroup
    ((4360, 136, 4500), {"gated": (257, 1, 1), "dx": (200, 14, 1), "dw": (200, 7, 1)}),
]
