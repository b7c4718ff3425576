"""Sizes at which neighbouring rows of attention over chosen pages are worked on together (from 1,024 pairs of a row and a key-value head on), for the
tests that need it to be so and the one that asks the library whether it is."""
import collections

Case = collections.namedtuple("Case", "heads lens news columns count")

# Sequences that begin inside a unit, one of a single row, one without rows, one with more rows than tokens
MIXED = Case(heads=4, lens=[700, 60, 300, 20, 30], news=[131, 1, 90, 0, 42], columns=48, count=9)
# Rows past max_new, rows of no sequence before and behind
PARTS = Case(heads=8, lens=[200, 90, 333], news=[60, 9, 71], columns=22, count=6)
# Lists so long that fewer rows fit a unit; a table so wide that fewer rows' bits do
LONG_LISTS = Case(heads=2, lens=[25_600], news=[512], columns=1600, count=1500)
WIDE_TABLE = Case(heads=2, lens=[256_000], news=[600], columns=16_000, count=40)
ALL = [(MIXED, g) for g in (1, 2, 4, 5)] + [(PARTS, g) for g in (1, 3)] + [(LONG_LISTS, 1), (WIDE_TABLE, 1)]
