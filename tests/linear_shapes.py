"""Shapes that between them take every kernel of splitee_linear_epilogue and splitee_grouped_linear with bfloat16
planes (tests/test_expert_plan.py holds them to it): ragged rows, odd N, K no multiple of a K tile."""


def _spread(rows, experts):
    """Uneven row counts: every third expert has twice its share, the last one the rest."""
    share = [2 if e % 3 == 0 else 1 for e in range(experts)]
    n = [rows * s // sum(share) for s in share]
    n[-1] += rows - sum(n)
    return n


# M, N, K
DENSE = [(1, 17, 72), (1, 17, 2032), (1, 4105, 2016), (829, 33, 200), (886, 17, 2376), (1655, 19, 72), (3770, 17, 2400), (5238, 1539, 72), (5424, 391, 1496), (5605, 69, 1240), (6352, 35, 1232), (6690, 129, 1680), (6863, 5433, 80), (7321, 5571, 208), (7340, 5745, 72), (7494, 399, 136), (7971, 1831, 560), (8711, 57, 72)]
# rows of each expert, N, K
GROUPED = [(_spread(r, e), n, k) for r, e, n, k in [(1, 2, 17, 80), (1, 2, 17, 2064), (57, 26, 163, 2008), (876, 2, 19, 2016), (1667, 3, 17, 200), (1803, 4, 17, 72), (2144, 7, 17, 2072), (7770, 32, 345, 144), (8546, 16, 49, 72), (8640, 11, 647, 144)]]
