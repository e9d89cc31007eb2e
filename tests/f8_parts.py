"""Sizes at which products of scaled 8-bit floats share sums between workgroups, as f8_ways.py has them: of every way and number of parts that the
library chooses, those that are not there.  Ends are short: of tiles, of the last part's four slabs, of the last slab."""

PARTS = [
    (2, 8, 19, 33, 8369, 0), (3, 8, 1083, 51, 8353, 0), (4, 2, 35, 8217, 6569, 0), (4, 8, 1037, 71, 8221, 0),
    (5, 2, 8281, 67, 5111, 0), (5, 8, 2083, 69, 8159, 0),
    (6, 2, 8681, 263, 23171, 0), (6, 4, 8241, 67, 7261, 0), (6, 8, 4279, 65, 15041, 0),
    (7, 2, 135, 11361, 8077, 0), (7, 4, 5445, 135, 5721, 0), (7, 8, 65, 4125, 10925, 0),
    (8, 2, 17335, 137, 8103, 0), (8, 4, 11275, 129, 9347, 0), (8, 8, 4237, 133, 15973, 0),
]


def slabs_of(k, parts):
    """Slabs of 128 of K that each of the workgroups has which share a sum: whole fours, dealt evenly from the front on, of which the last may be
    short."""
    slabs = -(-k // 128)
    fours = -(-slabs // 4)
    each = [fours // parts + (p < fours % parts) for p in range(parts)]
    ends = [min(4 * sum(each[:p + 1]), slabs) for p in range(parts)]
    return [b - a for a, b in zip([0] + ends, ends)]
