"""Sets of matrices that reach every tile width of Muon's products, none of them with a dimension that is a multiple of a tile.
A set is a list of (count, m, n)."""

# One word a value.  The second set of a pair has matrices of the same shapes on other tiles; the Gram matrices of both are single sums.
ONE_WORD_PAIRS = [([(1, 4001, 4001)], [(2, 4001, 4001)]),
                  ([(1, 2999, 3001)], [(2, 2999, 3001)]),
                  ([(1, 3001, 2999)], [(2, 3001, 2999)]),
                  ([(8, 701, 1003), (8, 1003, 701)], [(12, 701, 1003), (12, 1003, 701)]),
                  ([(32, 701, 1003)], [(8, 701, 1003)]),
                  ([(40, 699, 701)], [(8, 699, 701)]),
                  ([(24, 601, 1801)], [(9, 601, 1801)]),
                  ([(2, 1529, 3305), (2, 3305, 1529)], [(3, 1529, 3305), (3, 3305, 1529)]),
                  ([(6, 1529, 3305)], [(2, 1529, 3305)])]
# Few enough for 64 wide tiles and Gram matrices in partial sums.
ONE_WORD_SINGLES = [[(1, 1499, 1501)], [(1, 1501, 1499)], [(1, 1529, 3305)], [(1, 3305, 1529)]]
# Two words a value.
TWO_WORDS = [[(1, 4090, 4093)], [(2, 3001, 2999)], [(40, 699, 701)], [(2, 1529, 3305), (2, 3305, 1529)], [(8, 701, 1003), (8, 1003, 701)], [(1, 1501, 1499)],
             [(3, 1529, 3305)], [(1, 1529, 3305)]]


def shapes_of(groups):
    return [(m, n) for count, m, n in groups for _ in range(count)]
